"""fp64 oracle of the policy and preference losses over flat sequences of
tokens, and of gradient clipping: the definitions, sequence by sequence.

nll is the tokens' negative log-probability under the model; offsets [S + 1]
delimit the sequences; mask marks the trainable tokens.  Both losses return
(loss, w = d loss / d nll, extras).
"""
from __future__ import annotations

import math

import numpy as np

SUM, MEAN_TOKENS, MEAN_SEQS = 0, 1, 2
SIGMOID, HINGE, SQUARE = 0, 1, 2


def policy_loss(nll, old_nll, ref_nll, adv, mask, offsets, clip_low, clip_high, beta, scale, reduction):
    """Clipped policy loss with the KL estimator exp(e) - 1 - e, e = nll - ref_nll (ref_nll None: none).
    adv: one per sequence or per token.  A token is clipped by the fp32 difference old_nll - nll against the
    fp32 logarithms of the bounds.  Returns (loss, w, mean KL, share of clipped tokens)."""
    nll32, old32 = np.asarray(nll, np.float32), np.asarray(old_nll, np.float32)
    nll, old = np.asarray(nll, np.float64), np.asarray(old_nll, np.float64)
    T, S = len(nll), len(offsets) - 1
    on = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    hi, lo = np.float32(math.log1p(clip_high)), np.float32(math.log1p(-clip_low) if clip_low < 1 else -math.inf)
    n_all = int(on.sum())
    w = np.zeros(T)
    loss = kl_sum = 0.0
    clips = 0
    for s in range(S):
        t = [i for i in range(offsets[s], offsets[s + 1]) if on[i]]
        for i in t:
            A = float(adv[i] if len(adv) == T and len(adv) != S else adv[s])
            delta32 = old32[i] - nll32[i]
            rho = math.exp(old[i] - nll[i])
            if A > 0 and delta32 > hi:
                term, slope = -A * (1 + clip_high), 0.0
            elif A < 0 and delta32 < lo:
                term, slope = -A * (1 - clip_low), 0.0
            else:
                term, slope = -A * rho, A * rho
            clips += slope == 0.0 and A != 0.0
            if ref_nll is not None:
                e = nll[i] - float(ref_nll[i])
                term += beta * (math.expm1(e) - e)
                slope += beta * math.expm1(e)
                kl_sum += math.expm1(e) - e
            norm = scale * {SUM: 1.0, MEAN_TOKENS: 1.0 / n_all, MEAN_SEQS: 1.0 / (S * len(t))}[reduction]
            loss += norm * term
            w[i] = norm * slope
    n = max(n_all, 1)
    return loss, w, kl_sum / n, clips / n


def pref_loss(nll, ref_nll, mask, offsets, kind, mean_tokens, beta, margin, smoothing, scale):
    """Loss over pairs (sequences 2p, 2p + 1).  Returns (loss, w, rewards [2P])."""
    nll = np.asarray(nll, np.float64)
    T, P = len(nll), (len(offsets) - 1) // 2
    on = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    w, rewards, loss = np.zeros(T), np.zeros(2 * P), 0.0
    for p in range(P):
        R, at, share = [], [], []
        for c in (0, 1):
            a, b = offsets[2 * p + c], offsets[2 * p + c + 1]
            t = np.arange(a, b)[on[a:b]]
            v = -nll[t] if ref_nll is None else np.asarray(ref_nll, np.float64)[t] - nll[t]
            f = 1.0 / max(len(t), 1) if mean_tokens else 1.0
            R.append(math.fsum(v) * f)
            at.append(t)
            share.append(f)
        m = beta * (R[0] - R[1]) - margin
        if kind == SIGMOID:
            loss += (1 - smoothing) * np.logaddexp(0.0, -m) + smoothing * np.logaddexp(0.0, m)
            small = math.exp(-abs(m)) / (1 + math.exp(-abs(m)))  # of sigmoid(m) and sigmoid(-m)
            below, above = (small, 1 - small) if m >= 0 else (1 - small, small)
            slope = -(1 - smoothing) * below + smoothing * above
        elif kind == HINGE:
            loss += max(0.0, 1 - m)
            slope = -1.0 if m < 1 else 0.0
        else:
            loss += ((m - 0.5) / beta) ** 2
            slope = 2 * (m - 0.5) / beta ** 2
        for c, sign in ((0, -1.0), (1, 1.0)):
            w[at[c]] = sign * slope * beta * share[c] * scale / P
            rewards[2 * p + c] = beta * R[c]
    return loss * scale / P, w, rewards


def clip_grads(grads, max_norm):
    """(norm, coef, clipped tensors) of fp64 copies of `grads`."""
    grads = [np.asarray(g, np.float64) for g in grads]
    norm = math.sqrt(math.fsum(float((g * g).sum()) for g in grads))
    coef = max_norm / norm if math.isfinite(norm) and norm > max_norm else 1.0
    return norm, coef, [g * coef for g in grads]
