"""Quantized GBDT training hot path for NVIDIA B200: C-ABI CUDA library + thin Python binding.

`binding` exposes the calls of include/qgbdt.h; `synth` generates the seeded synthetic
workloads; `leaf_model` is a softmax classifier over the leaves of trained trees; `build` compiles
the library in-tree.  There is no CPU implementation here.
"""
