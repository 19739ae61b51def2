"""ONES evolutionary search (arXiv 2108.03645, Section 3.2) on MI355X: Python binding of
the C-ABI library plus the seeded synthetic clusters it is measured on, and the operators of a
scheduled job's training step (``train``)."""
from . import workloads  # noqa: F401

__all__ = ["workloads", "ones", "train"]


def __getattr__(name):
    if name in ("ones", "train"):
        import importlib
        return importlib.import_module("." + name, __name__)
    raise AttributeError(name)
