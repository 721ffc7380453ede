"""GCPSL hot path on MI355X (gfx950): HIP kernels behind a C ABI.

Submodules:
  gcpsl   binding of libgcpsl.so (include/gcpsl.h)
  driver  Alg. 2 loop over the binding (sample -> step -> periodic fuse)
  heads   a head of its own for every cluster, by the operators on tensors
  build   hipcc build of libgcpsl.so and _ops.so
"""
