"""Fused linear + cross-entropy (output projection and loss) for MI355X, in HIP, and the operators around it:
the residual's addition with RMSNorm in front, the global gradient norm and clipping behind."""
from .lce import (AdamConfig, HeadState, HeadStepTiming, LCEError, LinearCrossEntropy, PlanInfo,
                  RMSNormLinearCrossEntropy, auto_chunk_tokens, forward, forward_backward, forward_no_alloc, head_train_step,
                  host_adam_step, linear_cross_entropy, load_library, plan_info, rmsnorm_forward,
                  rmsnorm_forward_backward, rmsnorm_linear_cross_entropy, rmsnorm_workspace_size, timing_enable,
                  timing_read, workspace_size)
from .ops import (AddRMSNorm, add_rmsnorm, add_rmsnorm_backward, add_rmsnorm_forward, add_rmsnorm_quant,
                  add_rmsnorm_workspace_size, clip_grad_norm, clip_grad_norm_, grad_norm, grad_norm_workspace_size,
                  rmsnorm)

__all__ = ["AdamConfig", "AddRMSNorm", "HeadState", "HeadStepTiming", "LCEError", "LinearCrossEntropy", "PlanInfo",
           "RMSNormLinearCrossEntropy", "add_rmsnorm", "add_rmsnorm_backward", "add_rmsnorm_forward",
           "add_rmsnorm_quant", "add_rmsnorm_workspace_size", "auto_chunk_tokens", "clip_grad_norm", "clip_grad_norm_",
           "forward", "forward_backward", "forward_no_alloc", "grad_norm", "grad_norm_workspace_size",
           "head_train_step",
           "host_adam_step", "linear_cross_entropy", "load_library", "plan_info", "rmsnorm", "rmsnorm_forward",
           "rmsnorm_forward_backward", "rmsnorm_linear_cross_entropy", "rmsnorm_workspace_size", "timing_enable",
           "timing_read", "workspace_size"]
