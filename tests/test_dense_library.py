"""The types of the operators' C arguments are set on the library object that the calls go to, whichever was loaded before: without them
64-bit numbers are handed over as 32 bits."""


def test_types_are_those_of_the_library_in_use(monkeypatch):
    from paper_2305_01515_amd import dense, tbe
    first = dense._lib()
    assert first.tbe_scan_forward.argtypes and first.tbe_adamw_step.argtypes
    monkeypatch.setattr(tbe, "_lib", None)  # as where it is loaded a second time
    second = dense._lib()
    assert second is not first
    for name in [n for n in tbe.EXPORTS if n.startswith(("tbe_scan_", "tbe_bias_", "tbe_adamw_"))]:
        assert getattr(second, name).argtypes, name


def test_types_where_a_plan_is_closed_while_the_library_is_loaded(monkeypatch):
    from paper_2305_01515_amd import dense, tbe
    load, depth = tbe.lib, []
    monkeypatch.setattr(tbe, "_lib", None)
    monkeypatch.setattr(dense, "_ready", False)

    def lib():
        if not depth:  # a collected plan's close() asks for the library as well
            depth.append(1)
            dense._lib()
            monkeypatch.setattr(tbe, "_lib", None)
        return load()
    monkeypatch.setattr(tbe, "lib", lib)
    assert dense._lib().tbe_scan_step.argtypes
