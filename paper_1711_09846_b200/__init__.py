"""Lockstep Population Based Training on one B200: CUDA library + thin ctypes binding."""
from .binding import (EXPORTS, energy_fitness_static, grouped_gemm, selftest_bounded_wait, PbtError, Population, library_path, load_library, param_count,  # noqa: F401
                      spec_from_config)

_OPERATORS = ("AdapterProjection", "BlockNormGrads", "BlockNormOut", "Dropout", "GatedUnit", "GradientClip", "block_norm_backward", "block_norm_forward",
              "dropout_backward", "dropout_forward")


def __getattr__(name):
    """The operators, at their first use: they work on torch tensors, and the rest of the package is there without torch."""
    if name == "operators" or name in _OPERATORS:
        import importlib
        module = importlib.import_module(".operators", __name__)
        globals().update({n: getattr(module, n) for n in _OPERATORS})
        return module if name == "operators" else globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted({*globals(), *_OPERATORS, "operators"})
