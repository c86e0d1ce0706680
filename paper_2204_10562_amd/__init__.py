"""MI355X-native batched evaluation of synchronous-pipeline plans (arXiv 2204.10562).

`binding` wraps the C ABI of libpp.so (include/pp.h); `workloads` holds the seeded
synthetic inputs; `build` compiles the HIP sources.  `layer` wraps include/pp_layer.h: operators of the
layers that a stage runs (activations kept in 8 bits, linear layers in 4).
"""
