"""B200-native zero-value compression (ZVC) of activation maps and the
compressed offload / prefetch copy built on it (the cDMA method).

The library also has operators that make sparse maps: dropout whose mask is
never stored, and the gated feed-forward block with its backward pass.

``binding``   -- ctypes front end of the C-ABI CUDA library (``libcdma.so``).
``workloads`` -- seeded synthetic activation maps (inputs only).

Everything exists only as CUDA kernels for sm_100a; there is no CPU path.
"""
from . import binding, workloads  # noqa: F401

__all__ = ["binding", "workloads"]
