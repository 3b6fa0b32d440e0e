"""B200-native expert-cached MoE layer and the attention side of its decoder layer: CUDA library (csrc/), ctypes bindings and the seeded
synthetic workloads.  ``binding`` loads the shared library and fails loudly if it is missing."""
__all__ = ["attention", "binding", "build", "dense", "workload"]
