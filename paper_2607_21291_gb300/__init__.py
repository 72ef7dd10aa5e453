"""GB300-native depth-sparse forward of AdaDSF (Adaptive Depth Sparse Framework).

Submodules:
  adadsf  ctypes binding of the C ABI (include/adadsf.h) -> libadadsf.so
  serve   generation of sequences of different lengths from a paged cache, with sampling
  synth   seeded synthetic inputs and backbone shapes
  build   nvcc build of libadadsf.so for sm_103a
"""
