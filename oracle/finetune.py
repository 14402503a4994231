"""Oracle of the client's scoring and of its ends of a fine-tuning step (test infrastructure): the definitions in fp64, plain
numpy.  (Section 2.2, "Distributed fine-tuning": the client owns the loss and what is trained; the paper prints no formulas.)

Roundings of the forward pass count as the identity, as in oracle/backward.py.
"""
import numpy as np

from .backward import layernorm_backward

__all__ = ["softmax_rows", "logprobs", "distill", "lm_head_backward", "embed_backward"]


def softmax_rows(logits, temperature=1.0):
    """(q, log q) of every row; a row without a logit above -infinity: q = 0, log q = -infinity."""
    z = np.asarray(logits, np.float64) / temperature
    m = z.max(1, keepdims=True)
    m = np.where(m == -np.inf, 0.0, m)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.exp(z - m)
        s = e.sum(1, keepdims=True)
        logq = np.where(s == 0.0, -np.inf, z - m - np.log(s))
        q = np.where(s == 0.0, 0.0, e / s)
    return q, logq


def logprobs(logits, tokens, temperature=1.0, top_k=0):
    """(log probability of the tokens, entropy, top tokens, their log probabilities)."""
    V = logits.shape[1]
    q, logq = softmax_rows(logits, temperature)
    tokens = np.asarray(tokens)
    given = (tokens >= 0) & (tokens < V)
    lp = np.where(given, logq[np.arange(len(tokens)), np.where(given, tokens, 0)], 0.0)
    ent = -np.where(q == 0.0, 0.0, q * np.where(q == 0.0, 0.0, logq)).sum(1)
    top = np.argsort(-np.asarray(logits, np.float64), axis=1, kind="stable")[:, :top_k]
    return lp, ent, top, np.take_along_axis(logq, top, 1)


def distill(logits, ids, vals, temperature=1.0, loss_grad=None):
    """(loss per row, gradient of sum(loss_grad * loss))."""
    M, V = logits.shape
    q, logq = softmax_rows(logits, temperature)
    loss, grad = np.zeros(M), np.zeros((M, V))
    w = np.ones(M) if loss_grad is None else np.asarray(loss_grad, np.float64)
    for t in range(M):
        on = (ids[t] >= 0) & (ids[t] < V) & (vals[t] > -np.inf)
        if not on.any():
            continue
        if not (logits[t] > -np.inf).any():
            loss[t] = np.inf
            continue
        v = np.asarray(vals[t], np.float64)[on] / temperature
        p = np.exp(v - v.max())
        p /= p.sum()
        with np.errstate(invalid="ignore"):
            logp = np.where(p > 0.0, np.log(np.where(p > 0.0, p, 1.0)), 0.0)
            loss[t] = temperature ** 2 * np.where(p > 0.0, p * (logp - logq[t, ids[t][on]]), 0.0).sum()
        dense = q[t].copy()
        np.subtract.at(dense, ids[t][on], p)
        grad[t] = w[t] * temperature * dense
    return loss, grad


def lm_head_backward(hidden, grad_logits, E, gain, eps=1e-5):
    """Gradient of the hidden states, unrounded fp64."""
    da = np.asarray(grad_logits, np.float64) @ np.asarray(E, np.float64)
    return layernorm_backward(da, np.asarray(hidden, np.float64), np.asarray(gain, np.float64), eps)


def embed_backward(ids, grad_hidden, E, gain, eps=1e-5):
    """(different tokens ascending, gradient of their rows): the sum over positions of each position's own gradient."""
    ids = np.clip(ids, 0, E.shape[0] - 1)
    per = layernorm_backward(np.asarray(grad_hidden, np.float64), np.asarray(E, np.float64)[ids], np.asarray(gain, np.float64), eps)
    tokens, place = np.unique(ids, return_inverse=True)
    out = np.zeros((len(tokens), E.shape[1]))
    np.add.at(out, place.ravel(), per)
    return tokens, out
