"""MI355X (gfx950) hot path of DS-MPNN (arXiv 2402.15106).

Node sampling, radius-graph construction, the edge-conditioned
message-passing layer (forward and backward), the encoder, decoder and loss of
the hop loop, group norms, 8-bit activation checkpoints and attention within
packed sub-graphs as hand-written HIP kernels behind a C ABI (include/dsmpnn.h);
this package is the thin Python binding.
"""

from ._lib import (  # noqa: F401
    Dsmp, DsmpError, Graph, LayerDesc, layer_desc, load_library, LIB_PATH, EXPORTED, KERNEL_CLASSES,
    CAP_KNN, CAP_RANDOM, F32, BF16, ACT_IDENTITY, ACT_RELU, ACT_SILU, ACT_GELU, ATTR_CONCAT, ATTR_DIFF,
    ROTATE_HALF, ROTATE_INTERLEAVED, RotateDesc, rotate_desc, rotary_frequencies, AttentionDesc, attention_desc,
    GRAD_ACCUMULATE, GRAD_X_ACCUMULATE, MlpDesc, NormDesc, norm_desc, Checkpoint, EDGE_AUTO, EDGE_PER_EDGE, EDGE_AGGREGATE, OK, INVALID_ARG, CAPACITY, HIP_ERROR, UNSUPPORTED, WORKSPACE_TOO_SMALL,
)
from .hop import HopShapes, HopStep  # noqa: F401,E402
from .infer import SubdomainInference  # noqa: F401,E402
from .stack import CheckpointedStack, StackShapes  # noqa: F401,E402
from .attention import AttentionLayer, AttentionShapes  # noqa: F401,E402
