"""PWLQ breakpoint search + quantizer for MI355X (gfx950).

``paper_2002_00104_amd.pwlq`` is the binding (ctypes, and a module of C for calls of one
tensor) over the C-ABI library ``libpwlq.so`` (hand-written HIP).  ``paper_2002_00104_amd.block``
has the operators around the integer inner product in a transformer block: 8-bit rows, norms with gate and residual,
adapters, and their gradients.  ``paper_2002_00104_amd.attention`` has what lies between a block's projections: a paged cache of keys and
values, and attention over it.  ``paper_2002_00104_amd.synth`` holds the seeded input generators.  Nothing is imported eagerly so that the input
generators can be used without the GPU library being built.
"""

__all__ = ["attention", "block", "pwlq", "synth"]
