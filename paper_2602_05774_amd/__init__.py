"""VSD EM path scoring on AMD Instinct MI355X (gfx950).

The data-parallel hot path of Variational Speculative Decoding's EM draft
training, as hand-written HIP kernels behind a C ABI (include/vsd.h):
E-step sampling, path scoring with the oracle gate, ARW and CAR weights, the
weighted-likelihood loss and its gradient with respect to the draft logits,
from materialised logits or through a fused LM head (MFMA GEMM tiles consumed
in place), with shared rows per slot or with each family's own context rows.
Beside it, the base losses a trainer adds to that term: cross entropy and
distillation from a teacher's top logits, with their gradients (losses.py); and
what stands on either side of the step: a frozen head held in 8 bits (blocks.py),
draws under the deployed rule (draws.py), the gradients' norm and clipping
(gradients.py).
This package holds the kernels (csrc/), their build (build.py) and a thin
torch binding (vsd.py, losses.py, draws.py, blocks.py, gradients.py).
"""
from .blocks import BlockMatrix, block_product, product_workspace_bytes, quantize_blocks
from .draws import RowSamples, draw_workspace_bytes, sample_rows
from .gradients import GradClip, clip_gradients, grad_norm, norm_workspace_bytes
from .losses import (LossResult, TopLogits, cross_entropy, distill_loss, loss_workspace_bytes, top_logits,
                     top_workspace_bytes)
from .vsd import (VSD_CAR_LOGPROB, VSD_CAR_PROB, VSD_GRAD_ARW, VSD_GRAD_ARW_CAR, VSD_GRAD_BASIC, LmHead,
                  LmHeadGrad, Params, Problem, SampleResult, ScoreResult, VsdError, alloc_score_outputs, sample_paths,
                  sample_score_paths, sample_score_paths_static, sample_step, score_paths, score_paths_ctx, score_workspace_bytes,
                  score_workspace_needed_bytes, VerifyResult, verify_paths, weighted_loss_bwd, weighted_loss_bwd_ctx)

__all__ = ["LmHead", "LmHeadGrad", "Params", "Problem", "SampleResult", "ScoreResult", "VsdError", "alloc_score_outputs",
           "sample_paths", "sample_score_paths", "sample_score_paths_static", "score_paths", "score_workspace_bytes",
           "score_workspace_needed_bytes", "weighted_loss_bwd",
           "sample_step", "score_paths_ctx", "weighted_loss_bwd_ctx", "verify_paths", "VerifyResult",
           "cross_entropy", "distill_loss", "top_logits", "LossResult", "TopLogits", "loss_workspace_bytes",
           "top_workspace_bytes",
           "sample_rows", "RowSamples", "draw_workspace_bytes", "BlockMatrix", "quantize_blocks", "block_product",
           "product_workspace_bytes", "grad_norm", "clip_gradients", "GradClip", "norm_workspace_bytes",
           "VSD_GRAD_BASIC", "VSD_GRAD_ARW", "VSD_GRAD_ARW_CAR", "VSD_CAR_PROB", "VSD_CAR_LOGPROB"]
