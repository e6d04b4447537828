"""Cached embedding-bag training path (pooled lookup + sparse backward with
row-wise Adagrad through a set-associative LRU cache in HBM) for MI355X.

The HIP library binding lives in :mod:`paper_2305_01515_amd.tbe` and is loaded
on first attribute access, so that :mod:`paper_2305_01515_amd.synth` (seeded
input generators, no arithmetic of the method) can be imported on its own.
:mod:`paper_2305_01515_amd.dense` has operators for models on histories of looked-up rows.
"""

__all__ = ["tbe", "synth", "dense"]


def __getattr__(name):
    if name in ("tbe", "synth", "dense"):
        import importlib
        return importlib.import_module(f"{__name__}.{name}")
    raise AttributeError(name)
