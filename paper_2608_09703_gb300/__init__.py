"""GB300-native fused output stage of Matryoshka language-model suites.

For every nested sub-model the LM-head logits, the next-token cross-entropy
and the distillation term from the teacher sub-model (paper Eq. 2, Eq. 3),
forward and backward, in hand-written sm_103a kernels behind the C ABI of
include/mls.h.  ``binding`` is the Python face of that ABI.
"""
from .binding import (  # noqa: F401
    GradClip,
    HeadLogp,
    HeadLoss,
    LayerNorm,
    MLSError,
    PolicyLoss,
    PolicyProblem,
    Problem,
    SpecVerify,
    mls_get_status,
    mls_grad_clip,
    mls_grad_clip_workspace_size,
    mls_head_logp_bwd,
    mls_head_logp_fwd,
    mls_head_loss_bwd,
    mls_head_loss_fwd,
    mls_head_pairwise,
    mls_junction_bwd,
    mls_junction_fwd,
    mls_layer_norm_bwd,
    mls_layer_norm_fwd,
    mls_layer_norm_workspace_size,
    mls_logp_workspace_size,
    mls_policy_loss,
    mls_policy_workspace_size,
    mls_spec_verify,
    mls_spec_workspace_size,
    mls_strerror,
    mls_workspace_size,
)
