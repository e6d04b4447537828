"""Two places of a plan in the same memory would be stepped by two workgroups at once: refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_shared_memory():
    from paper_2305_01515_amd.dense import AdamW
    w, room = torch.nn.Parameter(torch.ones(40, 8).cuda()), torch.ones(1000).cuda()
    for params in ([w, torch.nn.Parameter(torch.ones(3).cuda()), w], [w, w.detach()[5:9]], [room[:501], room[500:]], [room, room[999:]]):
        with pytest.raises(ValueError, match="share"):
            AdamW(params)
    AdamW([room[:500], room[500:], room[1000:], room[1000:]])  # side by side, and empty ones
    states = {"m": torch.zeros(1024).cuda(), "v": torch.zeros(1024).cuda()}
    AdamW([room], states=states)
    with pytest.raises(ValueError, match="share"):
        AdamW([room], states=dict(states, v=states["m"]))
    half = torch.ones(64).cuda().bfloat16()
    copy = torch.ones(64).cuda()
    with pytest.raises(ValueError, match="share"):
        AdamW([half, half.clone()], master=[copy, copy])
    a, b = torch.ones(64).cuda(), torch.ones(64).cuda()
    opt = AdamW([a, b])
    opt.params[1] = a
    with pytest.raises(ValueError, match="share"):
        opt.step([torch.ones(64).cuda()] * 2)
    assert bool((a == 1).all()) and opt.step_count == 0
