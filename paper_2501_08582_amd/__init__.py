"""Sparsity-preserved LoRA linear (LoRS, arXiv 2501.08582) for AMD MI355X.

The compute lives in ``liblors.so`` (hand-written HIP kernels for gfx950 behind
the C ABI in ``include/lors.h``, ``include/lors_train.h`` and
``include/lors_block.h``).  Python modules:

``ops``    PyTorch-facing calls and the autograd ops: the layer, the gated block of
           two of them (imports torch)
``train``  the operators around the layer in a fine-tuning step: norm, dropout,
           embedding, preference loss, orthogonalised updates of the adapters,
           sampling (imports torch)
``finetune``  preference fine-tuning of a small sparse model with all of them
``_lib``   ctypes binding of the C ABI
``synth``  seeded synthetic inputs shaped like the paper's Llama projections
``costs``  flop / byte accounting
``build``  hipcc build of ``liblors.so``
"""

__all__ = ["ops", "train", "synth", "costs", "build"]
__version__ = "1.0.0"
