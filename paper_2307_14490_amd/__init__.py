"""MI355X-native training step of HUGE (KDD'23): skip-gram negative sampling
over (source_id, destination_id, co_counts) batches, in hand-written HIP
kernels behind the C ABI of ``include/huge.h``, the random-walk sampler
that produces those batches on the GPU, and the unsupervised evaluation of
the trained embeddings (edge SNR, distance percentiles, sampled recall), and
the training step of a softmax head on the embeddings (layer norm, the exact
softmax loss over all classes, AdamW) and what it answers with (RMS norm, rows
in 8 bits, log probabilities with the entropy and the most likely classes,
clipped gradients).

``binding`` is the ctypes layer, ``head`` and ``answer`` those of the softmax head's
operators;
``build`` compiles ``libhuge.so`` in-tree.
"""
from .binding import (  # noqa: F401
    EXPORTED,
    Evaluator,
    HUGE_NEG_ALIAS,
    HUGE_NEG_UNIFORM,
    HUGE_SCATTER_ATOMIC,
    HUGE_SCATTER_SORTED,
    HugeConfig,
    HugeError,
    HugeWalkConfig,
    Trainer,
    build_alias,
    cocount_weights,
    load,
    make_config,
    sample_walks,
    status_string,
    walk_config,
    workspace_bytes,
)
from .head import (  # noqa: F401
    AdamW,
    SoftmaxHead,
    SoftmaxLoss,
    layer_norm,
    layer_norm_backward,
)
from .answer import (  # noqa: F401
    Answers,
    LogProbs,
    Q8Rows,
    clip_grads,
    grad_norm,
    q8_rows,
    q8_values,
    rms_norm,
    rms_norm_backward,
)
