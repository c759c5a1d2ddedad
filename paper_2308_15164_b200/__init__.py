"""Delayed synchronous step of ABS-SGD (arXiv 2308.15164, Algorithm 1) on one B200.

The package holds:

* ``csrc/``      -- the sm_100a CUDA kernels and the C-ABI library built from them
                   (entry points declared in ``include/abs_sgd.h`` and ``include/abs_llm.h``),
* ``binding``    -- a ctypes binding with the same names (argument marshalling only),
* ``llm``        -- the operators of ``abs_llm.h`` on tensors (losses on logits, the residual join of a
                   transformer block, 8-bit activation checkpoints),
* ``llm_example`` -- a small model trained with them through the delayed synchronous step,
* ``workloads``  -- seeded synthetic input generators (no optimiser arithmetic).

Nothing here falls back to a CPU implementation: importing ``binding`` raises if the
shared library has not been built.
"""

__all__ = ["binding", "llm", "llm_example", "workloads", "build", "dist"]


def __getattr__(name):
    # Lazy sub-module import so that ``workloads`` can be used without the CUDA library.
    if name in __all__:
        import importlib

        return importlib.import_module(f"{__name__}.{name}")
    raise AttributeError(name)
