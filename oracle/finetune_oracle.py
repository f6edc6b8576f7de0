"""CPU oracle of the single operations of fine-tuning -- TEST INFRASTRUCTURE, not product code.

Plain fp64 NumPy statements of attention over one sequence with dropped probabilities, of dropout with bias and residual, and of
token log probabilities with entropy and top alternatives, each with its gradients, and of the counter-based generator that
the dropout masks come from.  Shares no code with the product.

Pins (tests/test_finetune_oracle.py): the generator's published test vectors, central differences for every gradient, closed forms."""
from __future__ import annotations

import numpy as np

MASK32 = np.uint64(0xFFFFFFFF)


def philox(c0, c1, c2, c3, seed, rounds=7):
    """Philox-4x32: arrays (or numbers) below 2^32 -> four uint64 arrays below 2^32."""
    c = [np.asarray(x, np.uint64) & MASK32 for x in (c0, c1, c2, c3)]
    c = list(np.broadcast_arrays(*c))
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64((seed >> 32) & 0xFFFFFFFF)]
    for r in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ k[0], p1 & MASK32, (p0 >> np.uint64(32)) ^ c[3] ^ k[1], p0 & MASK32]
        k = [(k[0] + np.uint64(0x9E3779B9)) & MASK32, (k[1] + np.uint64(0xBB67AE85)) & MASK32]
    return c


def drop_factors_attention(n, pair, p, seed, site):
    """[n, n] factors of one (sequence, head): 0 or 1 / kept share."""
    t = int(np.rint(p * 256))
    if t == 0:
        return np.ones((n, n))
    i, j = np.arange(n, dtype=np.uint64)[:, None], np.arange(n, dtype=np.uint64)[None, :]
    four = np.uint64(4)
    w = philox((i // four) << np.uint64(16) | (j // four), 0x80000000 | pair, site & 0xFFFFFFFF, (site >> 32) & 0xFFFFFFFF, seed)
    word = np.choose((i % four).astype(int) + np.zeros((n, n), int), w)
    byte = (word >> (np.uint64(8) * (j % four))) & np.uint64(255)
    return np.where(byte >= t, 256.0 / (256 - t), 0.0)


def drop_factors_rows(rows, n, p, seed, site):
    """[rows, n] factors of element-wise dropout."""
    t = int(np.rint(p * 65536))
    i, j = np.arange(rows, dtype=np.uint64)[:, None], np.arange(n, dtype=np.uint64)[None, :]
    w = philox(j // np.uint64(8), i, site & 0xFFFFFFFF, (site >> 32) & 0xFFFFFFFF, seed)
    word = np.choose(((j // np.uint64(2)) % np.uint64(4)).astype(int) + np.zeros((rows, n), int), w)
    half = (word >> (np.uint64(16) * (j % np.uint64(2)))) & np.uint64(65535)
    return np.where(half >= t, 65536.0 / (65536 - t), 0.0)


def attention(q, k, v, scale, causal, Z):
    """One sequence and head, [n, d] each.  Returns o, lse and what the backward needs."""
    n = q.shape[0]
    s = scale * (q @ k.T)
    if causal:
        s = np.where(np.arange(n)[None, :] <= np.arange(n)[:, None], s, -np.inf)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(-1, keepdims=True)
    P = e / l
    return (P * Z) @ v, (m + np.log(l))[:, 0], P


def attention_bwd(q, k, v, scale, Z, P, do):
    """dq, dk, dv, and dS (gradient of the scores) for error bounds."""
    dv = (P * Z).T @ do
    dP = (do @ v.T) * Z
    dS = P * (dP - (dP * P).sum(-1, keepdims=True))
    return scale * (dS @ k), scale * (dS.T @ q), dv, dS


def token_logprobs(x, ids, top):
    """logp, entropy, lse, top ids (by value, then lowest id) and their log probabilities of rows of logits."""
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(-1, keepdims=True)
        m0 = np.where(np.isfinite(m), m, 0.0)
        s = np.exp(x - m0).sum(-1, keepdims=True)
        lse = (m0 + np.log(s))[:, 0]
        lp = np.where(np.isneginf(x), -np.inf, x - lse[:, None])
        p = np.exp(lp)
        entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(-1)
    order = np.stack([np.lexsort((np.arange(x.shape[1]), -row)) for row in x])[:, :top] if top else np.zeros((x.shape[0], 0), int)
    logp = np.where(ids >= 0, lp[np.arange(len(ids)), np.maximum(ids, 0)], 0.0)
    return logp, entropy, lse, order, np.take_along_axis(lp, order, 1)


def token_logprobs_bwd(x, ids, g, h):
    """d logits from the gradients g of logp and h of entropy."""
    _, entropy, lse, _, _ = token_logprobs(x, ids, 0)
    with np.errstate(invalid="ignore"):
        lp = np.where(np.isneginf(x), -np.inf, x - lse[:, None])
    p = np.exp(lp)
    g = np.where(ids >= 0, g, 0.0)
    d = -p * (g[:, None] + h[:, None] * (np.where(p > 0, lp, 0.0) + entropy[:, None]))
    d[np.arange(len(ids)), np.maximum(ids, 0)] += g
    d[np.isneginf(lse)] = 0.0
    return d
