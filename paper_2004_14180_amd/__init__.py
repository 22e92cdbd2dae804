"""MI355X-native optimizer step of Quantized Adam with error feedback (arXiv 2004.14180).

The product is the gfx950 shared library ``libqadam_hip.so`` behind the C boundary declared in
``include/qadam.h``; :mod:`paper_2004_14180_amd.binding` is a thin argument-marshalling layer over
it with the same names, and :mod:`paper_2004_14180_amd.operators` that of the operators beside the step (AdamW over lists of tensors,
the gradients' norm, the embedding), :mod:`paper_2004_14180_amd.layers` that of layer norm, the product with weight codes and sampling.
PyTorch only provides device memory and streams.
"""
from .binding import (QADAM_IDENTITY, QAdam, QAdamConfig, QAdamError, library_path, load_library)  # noqa: F401
from .operators import AdamW, AdamWConfig, Embedding, GradNorm, adamw_state  # noqa: F401
from .layers import LayerNorm, Linear8, Sampler  # noqa: F401
