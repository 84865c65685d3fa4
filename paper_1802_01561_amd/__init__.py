"""libvtrace: the learner-side V-trace actor-critic step of IMPALA
(Espeholt et al., 2018) as hand-written HIP kernels for AMD Instinct MI355X.

The computation lives in ``libvtrace.so`` (C ABI in ``include/vtrace.h`` and, for
policies over a token vocabulary, ``include/vtrace_tokens.h`` and
``include/vtrace_parameters.h``); this package only loads it and marshals torch tensors
into it.
"""

from ._lib import LIB_PATH, VtraceError  # noqa: F401
from .binding import (  # noqa: F401
    HeadLossGrad,
    LossGrad,
    Workspace,
    vtrace_abi_version,
    vtrace_error_flag,
    vtrace_gather_logits,
    vtrace_head_loss_grad,
    vtrace_head_workspace_bytes,
    vtrace_loss_grad,
    vtrace_loss_grad_static,
    vtrace_max_elements,
    vtrace_targets,
    vtrace_workspace_bytes,
)
from .parameters import (  # noqa: F401
    QUINTIC,
    EmbedWorkspace,
    OrthogonalWorkspace,
    vtrace_orthogonalize,
    vtrace_orthogonalize_workspace_bytes,
    vtrace_vocab_embed,
    vtrace_vocab_embed_grad,
    vtrace_vocab_embed_grad_workspace_bytes,
)
from .tokens import (  # noqa: F401
    NO_TOKEN,
    ClipWorkspace,
    LogProbLossGrad,
    LogProbWorkspace,
    VocabGrad,
    VocabLogProbs,
    VocabWorkspace,
    vtrace_clip_grad_norm,
    vtrace_log_prob_loss_grad,
    vtrace_log_prob_workspace_bytes,
    vtrace_vocab_grad,
    vtrace_vocab_grad_workspace_bytes,
    vtrace_vocab_log_probs,
    vtrace_vocab_workspace_bytes,
)
