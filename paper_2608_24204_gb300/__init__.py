"""GB300-native batch-1 decoder forward pass (prefill + paged-KV greedy decode)
behind the C ABI of include/wici.h.  `wici` is the ctypes binding, `ops`
that of include/wici_ops.h (operators of a batched decode step, with `Rope`,
`PagedKV` and `KeyBounds`); `build` compiles libwici.so for sm_103a."""
from . import build, wici  # noqa: F401
from .wici import WiciModel, WiciError  # noqa: F401


def __getattr__(name):
    # ops needs torch at import; the rest of the package does not
    if name in ("ops", "Rope", "PagedKV", "KeyBounds"):
        import importlib
        ops = importlib.import_module(".ops", __name__)
        return ops if name == "ops" else getattr(ops, name)
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
