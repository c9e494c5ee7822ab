"""MI355X-native f16 GEMM (C = A B + C) and operators of transformer layers -- C-ABI library plus a thin binding.

`workloads` (input generators) imports nothing else from the package; the
binding in `binding` loads the HIP library on first use and raises if it has
not been built.  `expert_layer` runs the operators together in a feed-forward block with experts (needs torch).
"""
