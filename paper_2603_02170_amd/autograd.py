"""torch.autograd plumbing around the two calls of the library (no arithmetic of its own).

`sage_attention(Q, K, V, ...)` runs `sagebwd_fwd` and records what `sagebwd_bwd` needs, so that the
INT8 attention can stand where a model calls its attention (paper Sec. 5: SageBwd replaces the
attention of the training run, forward and backward).  Tensors are bf16 CUDA tensors, [B, H, N, d] or,
with `token_major`, [B, N, H, d]; K and V may have another length than Q.  The autograd node is native
(csrc/torch_host.cpp): the backward runs on the engine's thread without the interpreter.
"""
from __future__ import annotations

from . import binding


def sage_attention(Q, K, V, causal: bool = True, k_smooth: bool = True, q_smooth: bool = False, sm_scale: float = 0.0,
                   token_major: bool = False, share_quantized: bool = False, return_lse: bool = False):
    """O (and the log-sum-exp, in the smoothed frame) of INT8 attention, differentiable in Q, K, V.

    share_quantized: keep the forward's workspace until the backward and let it reuse psi(Q), psi(K)
    (Algorithm 2 takes them as inputs); costs that workspace's memory between the two calls."""
    O, L = binding._host().attention(Q, K, V, causal, k_smooth, q_smooth, sm_scale, token_major, share_quantized)
    return (O, L) if return_lse else O


def sage_rotary(Q, K, positions, inv_freq, sections=None, adjacent: bool = False, token_major: bool = True, inverse: bool = False):
    """Q and K (or Q alone, K = None) turned by their tokens' positions, differentiable in both.

    Q, K: bf16 [tokens, heads, d], [B, N, heads, d] or, without `token_major`, [B, heads, N, d]; any strides (those whose rows do not
    begin on 16 bytes are copied).  inv_freq: float32, one for every pair of channels that turns; the channels behind them pass.
    sections: how many of the frequencies go by each axis of `positions`, int32 or int64 [axes, tokens] (video: time, height, width);
    with one axis (the default) [tokens].  [axes, N] serves every batch.  adjacent: channel 2i turns with 2i + 1, else i with
    i + len(inv_freq).  inverse: by the negative angles.  Returns (Q, K) as new dense tensors.  inv_freq gets no gradient (one that
    wants it is refused).  A backward captured into a graph wants leaves that no eager graph still holds, as with any operator."""
    return binding._host().rotary(Q, K, positions, inv_freq, sections, adjacent, token_major, inverse)
