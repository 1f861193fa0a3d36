"""libgq: B200-native construction of GuidedQuant's guided layer objective.

``paper_2505_07004_b200.api`` is the ctypes binding of the C-ABI CUDA library
(``include/gq.h``); ``paper_2505_07004_b200.capture`` hooks it into PyTorch models, ``loss`` and
``quantized`` are the end loss and the quantised layer under autograd; ``synth`` draws seeded
synthetic layers.
"""
__version__ = "0.1.0"
