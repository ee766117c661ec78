"""B200-native CERAR coding pipeline (encode, ring rounds, decode) behind a C ABI.

`cerar`   thin ctypes binding of libcerar.so (argument marshalling only).
`training` the operators around the aggregation on torch tensors: 8-bit products with a scale per 128 values and
          their operands, gradient norm, AdamW over many tensors.
`inputs`  seeded synthetic gradient generators shaped like the paper's workloads.
`build`   compiles libcerar.so in-tree with nvcc for sm_100a.
"""
__all__ = ["cerar", "training", "inputs", "build"]
