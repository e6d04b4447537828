#!/usr/bin/env python3
"""Trains a small model on user histories with every part of the library: item rows looked up and trained through the cached embedding
path, pooled in order by a gated recurrence, attended to by the newest state with a learned bias by age, and the dense weights
stepped by AdamW with states in 8 bits.

    python examples/history_model.py [--steps 120] [--users 256] [--items 20000]

The data is synthetic: every item has a hidden sign, the label of a history is the sign of a sum over its items in which one counts
less the older it is.  What has to be learned is the items' signs (rows of the table) and how fast they fade (gates and bias).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

DIM, HEADS, LONGEST = 64, 4, 60


def batch(users, items, signs, g):
    """item of every row, offsets of the histories, time stamps [users, LONGEST], labels"""
    lengths = torch.randint(0, LONGEST + 1, (users,), generator=g)
    lengths[0] = LONGEST
    off = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)])
    item = torch.randint(0, items, (int(off[-1]),), generator=g)
    times = torch.randint(1, 5000, (users, LONGEST), generator=g).cumsum(1)
    age = lengths[:, None] - 1 - torch.arange(LONGEST)
    there = age >= 0
    padded = torch.zeros(users, LONGEST)
    padded[there] = signs[item]
    label = ((padded * 0.9 ** age.clamp(min=0) * there).sum(1) > 0).float()
    return item, off, lengths, times, there, label


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=120)
    ap.add_argument("--users", type=int, default=256)
    ap.add_argument("--items", type=int, default=20_000)
    a = ap.parse_args(argv)
    from paper_2305_01515_amd.dense import AdamW, RelativeBias, Scan, log_thresholds
    from paper_2305_01515_amd.tbe import TBE, pinned_empty

    g = torch.Generator().manual_seed(1)
    signs = torch.randint(0, 2, (a.items,), generator=g) * 2.0 - 1
    most = a.users * LONGEST
    rows, state = pinned_empty((a.items, DIM), torch.float32), pinned_empty((a.items,), torch.float32)
    rows.normal_(std=0.1, generator=g)
    state.zero_()
    table = TBE([rows], [state], [a.items // 4], 32, max_batch=most, max_lookups=most)
    scan = Scan(DIM, torch.float32, max_bags=a.users, max_rows=most)
    thresholds = log_thresholds(16, 300_000)
    bias = RelativeBias(HEADS, thresholds)

    def weight(*shape, std):
        return torch.nn.Parameter((torch.randn(*shape, generator=g) * std).cuda())
    gate_w, gate_b = weight(DIM, DIM, std=0.05), torch.nn.Parameter(torch.full((DIM,), 1.0, device="cuda"))
    query_w, key_w, out_w, out_b = weight(DIM, DIM, std=0.1), weight(DIM, DIM, std=0.1), weight(2 * DIM, std=0.1), torch.nn.Parameter(torch.zeros(1, device="cuda"))
    bias_table = torch.nn.Parameter(torch.zeros(bias.buckets, HEADS, device="cuda"))
    dense = [gate_w, gate_b, query_w, key_w, out_w, out_b, bias_table]
    opt = AdamW(dense, lr=2e-3, weight_decay=[0.01 if p.dim() > 1 else 0.0 for p in dense], state_bits=8, seed=1)

    losses = []
    for step in range(a.steps):
        item, off, lengths, times, there, label = batch(a.users, a.items, signs, g)
        n = item.numel()
        item, off, lengths, times, there, label = (t.cuda() for t in (item, off, lengths, times, there, label))
        one_each = torch.arange(n + 1, device="cuda")  # a lookup a history row: bags of one
        x = table.forward(item, one_each).requires_grad_()
        y, newest = scan(x, x @ gate_w + gate_b, off)

        keys = torch.zeros(a.users, LONGEST, DIM, device="cuda").masked_scatter(there[..., None], y)
        heads = lambda t: t.view(a.users, -1, HEADS, DIM // HEADS).transpose(1, 2).contiguous()  # noqa: E731
        q, k, v = heads(newest @ query_w), heads(keys @ key_w), heads(keys)
        scores = q @ k.transpose(2, 3).contiguous()
        now = times.gather(1, (lengths - 1).clamp(min=0)[:, None])
        lowest = torch.finfo(torch.float32).min  # a history without a row: equal weights of keys that are all zero
        scores = bias(bias_table, scores, scale=(DIM // HEADS) ** -0.5, q_pos=now, k_pos=times, key_lengths=lengths, mask_value=lowest)
        pooled = (scores.softmax(-1) @ v).transpose(1, 2).reshape(a.users, DIM)

        logit = torch.cat([newest, pooled], 1) @ out_w + out_b
        loss = torch.nn.functional.binary_cross_entropy_with_logits(logit, label)
        for p in dense:
            p.grad = None
        loss.backward()
        table.backward_update(x.grad.contiguous() * a.users, lr=0.05, eps=1e-8)  # the rows' own rate: a mean's gradient is small
        opt.step()
        losses.append(float(loss.detach()))
        if step % 20 == 19:
            print(f"step {step + 1}: loss {sum(losses[-20:]) / 20:.4f}", flush=True)
    scan.check()
    table.flush()
    table.close()
    return losses


if __name__ == "__main__":
    main()
