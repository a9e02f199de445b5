"""The distillation objective from a teacher's stored top logits as a differentiable torch call.

    ids, values, rest = hdf.top_logits(teacher_logits, K, temperature=T)      # once, stored
    loss, kl, ce = distill_loss(student_logits, ids, values, rest, labels, B=B, temperature=T)
    loss[2].backward()

Both directions run in libhdf's kernels; this module only connects them to autograd.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import hdf


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, student, ids, values, rest, labels, B, temperature, alpha):
        if student.dim() == 2 and student.shape[1] > 1 and student.stride(1) != 1:
            student = student.contiguous()
        kl, ce, loss, saved = hdf.distill_forward(student, ids, values, rest, labels, B=B,
                                                  temperature=temperature, alpha=alpha)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(student, ids, labels, saved)
        ctx.settings = dict(B=B, temperature=temperature, alpha=alpha)
        return loss, kl, ce

    @staticmethod
    @once_differentiable
    def backward(ctx, g_loss, g_kl, g_ce):
        if not ctx.needs_input_grad[0] or (g_loss is None and g_kl is None and g_ce is None):
            return (None,) * 8
        student, ids, labels, saved = ctx.saved_tensors
        g = [x if x is None else x.to(torch.float32).contiguous() for x in (g_loss, g_kl, g_ce)]
        d = hdf.distill_backward(student, ids, labels, saved, grad_loss=g[0], grad_kl=g[1],
                                 grad_ce=g[2], **ctx.settings)
        return (d,) + (None,) * 7


def distill_loss(student_logits: torch.Tensor, teacher_ids: torch.Tensor,
                 teacher_logits: torch.Tensor, teacher_rest: Optional[torch.Tensor] = None,
                 labels: Optional[torch.Tensor] = None, *, B: int, temperature: float = 1.0,
                 alpha: float = 0.1):
    """(loss [3] = L_KL, L_CE, L_CE + alpha L_KL; kl [n_seq, P]; ce [n_seq, B-1] or None), each
    differentiable with regard to student_logits alone.  Arguments as hdf.distill_forward.  To
    capture a training step, call hdf.distill_forward and hdf.distill_backward themselves."""
    return _DistillLoss.apply(student_logits, teacher_ids, teacher_logits, teacher_rest, labels, B,
                              temperature, alpha)
