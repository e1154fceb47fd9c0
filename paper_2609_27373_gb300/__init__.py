"""WISE attention hot path on GB300 (sm_103a).

The compute path is the C-ABI library libwise.so built from csrc/:
hand-written CUDA kernels for dense causal attention with a fused block-mass
epilogue, support selection and support-restricted sparse attention, and for
answering with the model afterwards a paged cache, attention over prefixes
that requests share, and the verification of drafted tokens.
`paper_2609_27373_gb300.wise` is the thin ctypes binding with the same names
as the C entry points; `serve` has the cache as a class; `synth` draws seeded
synthetic inputs.
"""
