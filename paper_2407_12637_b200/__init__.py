"""B200-native quantized backward pass of arXiv 2407.12637 (INT4 fixed-point training).

`lbt`     -- thin ctypes binding of the C-ABI CUDA library (argument marshalling only).
`lm`      -- layers of a transformer's residual block: 8-bit linear layer, norm / gate / residual, AdamW.
`block_train` -- example: a stack of such blocks trained with them (`python -m paper_2407_12637_b200.block_train`).
`synth`   -- seeded synthetic inputs shaped like the paper's CNN workloads.
`shapes`  -- the layer shapes of the benchmark configurations.
`build`   -- compiles the CUDA library for sm_100a.

Nothing here imports a CPU implementation of the method; the CUDA library is
loaded on first use of `lbt` and its absence is an error.
"""
__all__ = ["lbt", "lm", "synth", "shapes", "build"]
