"""B200-native implementation of SPRINTER's verification-and-replacement step.

``sprinter_verify``, ``replace_sample`` and ``sd_verify`` are thin wrappers over the C ABI
of ``libsprinter.so`` (CUDA kernels for sm_100a), and so are the calls that fit a draft head and a
verifier (``head_loss``, ``verifier_labels_head``, ``hidden_pack8``, ``verifier_train_step8`` ...) and the
calls of the target's pass over drafted tokens that come before the check (``cache_append``, ``tree_attention``,
``logits_rules``); ``workloads`` draws the synthetic inputs.
"""
from . import workloads  # noqa: F401
from .binding import (Arena, host_arena_bytes, replace_sample_host, sd_verify_host,  # noqa: F401
                      replace_sample_static, set_stage_events, sprinter_verify_host)
from .binding import (BF16, F32, PATH_AUTO, PATH_SIMT, PATH_TENSOR, SprinterError, Workspace,  # noqa: F401
                      lib, replace_sample, sd_verify, sprinter_simulate, sprinter_step, sprinter_verify, workspace_bytes)
from .binding import (OP_HEAD_LOSS, OP_HEAD_LOSS_GRAD, OP_VERIFIER_LABELS_HEAD, OP_VERIFIER_TRAIN8,  # noqa: F401
                      head_loss, head_loss_grad, hidden_pack8, hidden_unpack8, pack8_pitch, verifier_labels_head,
                      verifier_train_step8)
from .binding import (OP_CACHE_APPEND, OP_LOGITS_RULES, OP_TREE_ATTENTION, cache_append, logits_rules,  # noqa: F401
                      tree_attention)
