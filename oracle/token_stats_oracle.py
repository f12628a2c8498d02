"""CPU oracle for the token statistics of rows of hidden states under an output matrix, and for their gradient.
TEST INFRASTRUCTURE ONLY.

Only tests/, __graft_entry__.smoke() and the cpu_baseline leg of bench.py may import this module.  It shares no code with the
HIP library and never imports it.  Plain float64 numpy, one row at a time.

Forward, with l = W h_t, z = l / T and p = softmax(z):

    lse_t = log sum_v exp z_v,   logprob_t = z_y - lse_t (0 without a target),   entropy_t = - sum_v p_v log p_v
    alternatives: the k entries of largest l, equal ones by lower id, NaN last

Backward of a scalar loss with dL/dlogprob_t = g_t and dL/dentropy_t = e_t: since d log p_y / dz_v = [v = y] - p_v and
d entropy / dz_v = - p_v (log p_v + entropy),

    dL/dl_v = (g_t ([v = y] - p_v) - e_t p_v (log p_v + entropy_t)) / T,   dL/dh_t = W^T dL/dl,   dL/dW = sum_t dL/dl h_t^T

Pins (tests/test_oracle_token_stats_pins.py): central differences, reverse-mode differentiation of torch's log-softmax in
float64, closed forms (equal logits, one sure token), ties.
"""
from __future__ import annotations

import numpy as np

F64 = np.float64


def token_stats(hidden, weight, targets, temperature, top_k=0):
    """float64 dict of logprobs, entropy, lse [T] and, with top_k, top_ids, top_logprobs [T, top_k]."""
    h, w = np.asarray(hidden, F64), np.asarray(weight, F64)
    T, V = h.shape[0], w.shape[0]
    out = dict(logprobs=np.zeros(T), entropy=np.zeros(T), lse=np.zeros(T))
    if top_k:
        out.update(top_ids=np.zeros((T, top_k), np.int64), top_logprobs=np.zeros((T, top_k)))
    for t in range(T):
        logits = w @ h[t]
        z = logits / temperature
        m = z.max()
        lse = m + np.log(np.exp(z - m).sum())
        logp = z - lse
        p = np.exp(logp)
        out["lse"][t] = lse
        out["entropy"][t] = -(p[p > 0] * logp[p > 0]).sum()
        if 0 <= targets[t] < V:
            out["logprobs"][t] = logp[targets[t]]
        if top_k:
            order = sorted(range(V), key=lambda v: (np.isnan(logits[v]), -logits[v], v))[:top_k]
            out["top_ids"][t], out["top_logprobs"][t] = order, logp[order]
    return out


def token_stats_backward(hidden, weight, targets, d_logprobs, d_entropy, temperature):
    """(d_hidden, d_weight, dl): float64 gradients and the gradient of the logits that they come from."""
    h, w = np.asarray(hidden, F64), np.asarray(weight, F64)
    T, V = h.shape[0], w.shape[0]
    dl = np.zeros((T, V))
    for t in range(T):
        z = w @ h[t] / temperature
        logp = z - z.max()
        logp -= np.log(np.exp(logp).sum())
        p = np.exp(logp)
        if 0 <= targets[t] < V:
            dl[t] -= d_logprobs[t] * p
            dl[t, targets[t]] += d_logprobs[t]
        if d_entropy is not None:
            plogp = np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0)
            dl[t] -= d_entropy[t] * (plogp - p * plogp.sum())
    dl /= temperature
    return dl @ w, dl.T @ h, dl
