"""AdaCGD hot path for MI355X: hand-written HIP kernels behind a C ABI.

`workloads` (seeded synthetic inputs) imports without the native library;
`engine` loads the library on first use and raises if it has not been built, and so does
`layers`, the operators of a model whose gradients are passed to the engine.
"""
__all__ = ["workloads", "engine", "layers"]
