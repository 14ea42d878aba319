"""Performance cases of the operators around preference and policy fine-tuning
of an adapted model, each one pass through one operator:

  decode  adapted projections with 4-bit weights for 1 to 16 tokens
          (lora_decode_q4): the step that samples an answer
  policy  the clipped policy loss with its KL term, and the gradient of the
          hidden states (lora_policy_fwd_bwd)
  pref    the loss over pairs of a chosen and a rejected answer, and the
          gradient of the hidden states (lora_pref_fwd_bwd)
  clip    the global norm of many gradient tensors, and their clipping
          (lora_clip_grads)

With `own` unset the operators run in a plain form of elementary torch
operations in 32 bits; with `own` set through the library.  Sizes are those of
the Llama-3.2-3B- and Qwen-2.5-3B-shaped layers of
paper_2606_19528_gb300/workloads.py, or generic.
"""
from __future__ import annotations

import math

import torch

own = False

LLAMA = {"q": (3072, 3072), "k": (3072, 1024), "v": (3072, 1024), "o": (3072, 3072), "gate": (3072, 8192),
         "up": (3072, 8192), "down": (8192, 3072)}


def _dims(text):
    return [tuple(int(v) for v in p.split("x")) for p in text.split(",")]


def listed():
    return [
        # the smallest adapted linear of the configurations, one token: bound by latency
        dict(op="decode", name="decode_T1_256x256_r8", T=1, dims="256x256", r=8),
        # sampling one answer: the q, k and v projections of a layer for one token
        dict(op="decode", name="decode_T1_llama_qkv_r16", T=1, dims="3072x3072,3072x1024,3072x1024", r=16),
        # five answers sampled side by side, a large rank: gate and up of the wider layer
        dict(op="decode", name="decode_T5_qwen_gate_up_r64", T=5, dims="2048x11008,2048x11008", r=64),
        # sixteen answers side by side: the frozen head, every logit
        dict(op="decode", name="decode_T16_head_128256", T=16, dims="3072x128256", r=0),
        # a test-sized policy step: four short answers of odd lengths, no reference model
        dict(op="policy", name="policy_S4_T61_d256", S=4, T=61, d=256, prompt=0.2, kl=False, reduction="seqs",
             per_token=False),
        # a group of sixteen answers to one prompt, one advantage each, with the KL term
        dict(op="policy", name="policy_S16_T4096_d3072", S=16, T=4096, d=3072, prompt=0.3, kl=True,
             reduction="tokens", per_token=False),
        # a large batch with an advantage per token (from a value model)
        dict(op="policy", name="policy_S64_T49152_d2048", S=64, T=49152, d=2048, prompt=0.25, kl=True,
             reduction="seqs", per_token=True),
        # one short pair: bound by latency
        dict(op="pref", name="pref_P1_T48_d256", P=1, T=48, d=256, prompt=0.3, ref=True, kind="sigmoid",
             mean_tokens=False),
        # the ordinary step: 32 pairs of some hundred tokens
        dict(op="pref", name="pref_P32_T16384_d3072", P=32, T=16384, d=3072, prompt=0.4, ref=True, kind="sigmoid",
             mean_tokens=False),
        # the adapters on q and v of one layer, as the fine-tuning method places them
        dict(op="clip", name="clip_qv_1layer_r16", layers=1, dims="3072x3072,3072x1024", r=16, half=0, frac=0.5),
        # tensors of odd sizes, some of them in 16 bits (other parameters trained beside the adapters)
        dict(op="clip", name="clip_ragged_5layers_r7", layers=5, dims="1001x777,519x2049,64x33", r=7, half=3,
             frac=0.5),
        # every adapter of a 28-layer model
        dict(op="clip", name="clip_llama_28layers_r16", layers=28,
             dims=",".join("%dx%d" % v for v in LLAMA.values()), r=16, half=0, frac=0.5),
    ]


# ---------------------------------------------------------------- drawn cases
def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + step - 1)))
    return max(lo, min(hi, int(v) // step * step))


def draw(rng):
    op = rng.choice(["decode", "policy", "pref", "clip"])
    if op == "decode":
        n = rng.choice([1, 1, 2, 3, 7])
        K = _log(rng, 64, 12288, 64)
        room = 128256 * 2048 // (K * n)
        dims = ",".join("%dx%d" % (K, max(1, min(_log(rng, 16, 131072), room))) for _ in range(n))
        return dict(op=op, T=rng.randint(1, 16), dims=dims, r=rng.choice([0, 4, 8, 13, 16, 32, 64, 128]))
    if op in ("policy", "pref"):
        d = _log(rng, 64, 4096, 8)
        seqs = _log(rng, 1, 128)
        T = min(_log(rng, 2, 65536), 49152 * 2048 // d)
        if op == "policy":
            return dict(op=op, S=seqs, T=T, d=d, prompt=round(rng.uniform(0.0, 0.6), 2), kl=rng.random() < 0.7,
                        reduction=rng.choice(["sum", "tokens", "seqs"]), per_token=rng.random() < 0.4)
        return dict(op=op, P=(seqs + 1) // 2, T=T, d=d, prompt=round(rng.uniform(0.0, 0.6), 2),
                    ref=rng.random() < 0.8, kind=rng.choice(["sigmoid", "hinge", "square"]),
                    mean_tokens=rng.random() < 0.4)
    r = rng.choice([4, 7, 8, 16, 32, 64])
    dims = ",".join("%dx%d" % (_log(rng, 64, 11008), _log(rng, 64, 11008)) for _ in range(rng.randint(1, 7)))
    most = 24_000_000 // (r * sum(sum(v) for v in _dims(dims)))
    return dict(op=op, layers=max(1, min(_log(rng, 1, 40), most)), dims=dims, r=r, half=rng.choice([0, 0, 1, 4]),
                frac=rng.choice([0.2, 0.5, 0.9, 1.5]))


# ---------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _proj(g, T, K, N, r):
    """4-bit codes of a weight of variance 1 / K: 16 levels over about +-2.5 standard deviations."""
    sd = K ** -0.5
    s = torch.empty(N, K // 64, device="cuda").uniform_(0.25, 0.41, generator=g) * sd
    b = -7.5 * s + torch.empty_like(s).uniform_(-0.2, 0.2, generator=g) * sd
    p = {"K": K, "N": N,
         "codes": torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8),
         "params": torch.stack([s, b], dim=-1).to(torch.bfloat16).contiguous(),
         "y": torch.empty(T, N, device="cuda", dtype=torch.bfloat16)}
    if r:
        p["A"] = (torch.rand(r, K, generator=g, device="cuda") * 2 - 1).mul_(sd).to(torch.bfloat16)
        p["B"] = _normal(g, N, r, std=0.02)
    return p


def _tokens(g, case, seqs):
    """Answers of uneven lengths (also empty ones), a prompt first in each, its positions not trained."""
    T, d = case["T"], case["d"]
    cuts = torch.randint(0, T + 1, (seqs - 1,), generator=g, device="cuda").sort().values
    edge = torch.tensor([0, T], device="cuda")
    offsets = torch.cat([edge[:1], cuts, edge[1:]])
    lens = offsets[1:] - offsets[:-1]
    at = torch.arange(T, device="cuda")
    seq = torch.searchsorted(offsets, at, right=True) - 1
    mask = at - offsets[seq] >= (lens[seq].double() * case["prompt"]).floor()
    zero = torch.zeros(T, device="cuda")
    nll = torch.where(mask, _normal(g, T, dtype=torch.float32).square() * 1.1 + 0.01, zero)
    dh = _normal(g, T, d, std=d ** -0.5) * mask[:, None]
    return {"T": T, "d": d, "seqs": seqs, "offsets": offsets.int(), "longest": int(lens.max()),
            "mask": mask.to(torch.uint8), "nll": nll, "dh_nll": dh.to(torch.bfloat16).contiguous(),
            "ref_nll": torch.where(mask, (nll + _normal(g, T, std=0.15, dtype=torch.float32)).abs(), zero),
            "loss": torch.empty(1, device="cuda"), "token_weight": torch.empty(T, device="cuda"),
            "dh": torch.empty(T, d, device="cuda", dtype=torch.bfloat16)}


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "decode":
        T, r, scale = case["T"], case["r"], 2.0
        projs = [_proj(g, T, K, N, r) for K, N in _dims(case["dims"])]
        # projections of one call read the same activation
        return {"op": op, "T": T, "r": r, "scale": scale, "projs": projs, "x": _normal(g, T, projs[0]["K"])}
    if op == "policy":
        s = _tokens(g, case, case["S"])
        T = s["T"]
        s.update(op=op, low=0.2, high=0.28, beta=0.04, scale=1.0, reduction=case["reduction"], kl=case["kl"],
                 per_token=case["per_token"],
                 adv=_normal(g, T if case["per_token"] else s["seqs"], dtype=torch.float32),
                 old_nll=(s["nll"] + _normal(g, T, std=0.15, dtype=torch.float32) * s["mask"]).abs(),
                 stats=torch.empty(2, device="cuda"))
        return s
    if op == "pref":
        s = _tokens(g, case, 2 * case["P"])
        s.update(op=op, kind=case["kind"], mean_tokens=case["mean_tokens"], ref=case["ref"], beta=0.1, margin=0.05,
                 smoothing=0.1 if case["kind"] == "sigmoid" else 0.0, scale=1.0,
                 rewards=torch.empty(s["seqs"], device="cuda"))
        return s
    sizes = [r * n for r in [case["r"]] for K, N in _dims(case["dims"]) for n in (K, N)] * case["layers"]
    half = min(case["half"], len(sizes) - 1)
    kinds = [torch.bfloat16] * half + [torch.float32] * (len(sizes) - half)
    grads = [_normal(g, n, std=10.0 ** (i % 5 - 4), dtype=t) for i, (n, t) in enumerate(zip(sizes, kinds))]
    std = math.sqrt(sum(n * 10.0 ** (2 * (i % 5 - 4)) for i, n in enumerate(sizes)))
    # the clipped gradients go into the buffers that a data-parallel exchange or an optimizer takes whole
    packed = [torch.empty(sum(sizes[:half]), device="cuda", dtype=torch.bfloat16),
              torch.empty(sum(sizes[half:]), device="cuda")]
    return {"op": op, "grads": grads, "half": half, "packed": packed, "max_norm": case["frac"] * std,
            "norm": torch.empty(1, device="cuda"), "coef": torch.empty(1, device="cuda")}


# ---------------------------------------------------------------- one pass
def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["op"]](state)


def _plain_weight(p):
    """W = bf16(s q + b): the weight that the 4-bit form stands for."""
    N, K = p["N"], p["K"]
    shift = torch.arange(4, device="cuda", dtype=torch.int32)[:, None] * 4 + torch.tensor([0, 16], device="cuda",
                                                                                          dtype=torch.int32)
    q = (p["codes"].view(torch.int32)[:, :, None, None] >> shift) & 15  # [N, K / 8, 4, 2]
    sb = p["params"].float()
    q = q.view(N, K // 64, 64).float()
    return (sb[:, :, :1] * q + sb[:, :, 1:]).to(torch.bfloat16).float().view(N, K)


def _plain_proj(state, p):
    x = state["x"].float()
    y = x @ _plain_weight(p).T
    if state["r"]:
        y = y + (state["scale"] * (x @ p["A"].float().T)) @ p["B"].float().T
    return y.to(torch.bfloat16)


def _plain_decode(state):
    return [_plain_proj(state, p) for p in state["projs"]]


def _plain_rows(w, dh):
    """Each row times its weight; rows of weight zero are zero."""
    out = w[:, None] * dh.float()
    return torch.where(w[:, None] == 0, torch.zeros_like(out), out).to(torch.bfloat16)


def _plain_segments(state, values):
    """Sums over the sequences of `values` [T]."""
    off = state["offsets"].long()
    at = off[:-1, None] + torch.arange(state["longest"], device="cuda")
    inside = at < off[1:, None]
    v = values[at.clamp(max=state["T"] - 1)]
    return torch.where(inside, v, torch.zeros_like(v)).sum(dim=1)


def _plain_sequence(state):
    off = state["offsets"].long()
    return torch.repeat_interleave(torch.arange(state["seqs"], device="cuda"), off[1:] - off[:-1],
                                   output_size=state["T"])


def _plain_policy(state):
    on = state["mask"] != 0
    zero = torch.zeros_like(state["nll"])
    seq = _plain_sequence(state)
    adv = state["adv"] if state["per_token"] else state["adv"][seq]
    delta = state["old_nll"] - state["nll"]
    high = torch.tensor(math.log1p(state["high"]), device="cuda", dtype=torch.float32)
    low = torch.tensor(math.log1p(-state["low"]), device="cuda", dtype=torch.float32)
    up, down = (adv > 0) & (delta > high), (adv < 0) & (delta < low)
    ratio = torch.exp(delta)
    bound = torch.where(up, 1 + state["high"] + zero, torch.where(down, 1 - state["low"] + zero, ratio))
    clipped = up | down
    loss = -adv * bound
    w = torch.where(clipped, zero, adv * ratio)
    kl = zero
    if state["kl"]:
        e = state["nll"] - state["ref_nll"]
        grad = torch.expm1(e)
        kl = grad - e
        loss = loss + state["beta"] * kl
        w = w + state["beta"] * grad
    n = on.sum().float()
    if state["reduction"] == "sum":
        norm = torch.ones_like(zero)
    elif state["reduction"] == "tokens":
        norm = (1 / n).expand_as(zero)
    else:
        norm = (1 / (state["seqs"] * _plain_segments(state, on.float())))[seq]
    norm = norm * state["scale"]
    w = torch.where(on, w * norm, zero)
    stats = torch.stack([torch.where(on, kl, zero).sum() / n, (clipped & on).sum().float() / n])
    return {"loss": torch.where(on, loss * norm, zero).sum().view(1), "stats": stats, "token_weight": w,
            "dh": _plain_rows(w, state["dh_nll"])}


def _plain_pref(state):
    on = state["mask"] != 0
    zero = torch.zeros_like(state["nll"])
    beta = state["beta"]
    ratio = torch.where(on, (state["ref_nll"] if state["ref"] else zero) - state["nll"], zero)
    score = _plain_segments(state, ratio)
    share = torch.ones_like(score)
    if state["mean_tokens"]:
        share = 1 / _plain_segments(state, on.float()).clamp(min=1)
        score = score * share
    m = beta * (score[0::2] - score[1::2]) - state["margin"]
    if state["kind"] == "sigmoid":
        ls = state["smoothing"]
        tail = torch.log1p(torch.exp(-m.abs()))  # log(1 + e^-|m|)
        loss = (1 - ls) * (tail + (-m).clamp(min=0)) + ls * (tail + m.clamp(min=0))
        slope = -(1 - ls) / (1 + torch.exp(m)) + ls / (1 + torch.exp(-m))
    elif state["kind"] == "hinge":
        loss = (1 - m).clamp(min=0)
        slope = -(m < 1).float()
    else:
        loss = ((m - 0.5) / beta).square()
        slope = 2 * (m - 0.5) / (beta * beta)
    per = slope * (beta * state["scale"] / m.numel())
    w = (torch.stack([-per, per], dim=1).view(-1) * share)[_plain_sequence(state)]
    w = torch.where(on, w, zero)
    return {"loss": (loss.sum() * (state["scale"] / m.numel())).view(1), "rewards": beta * score, "token_weight": w,
            "dh": _plain_rows(w, state["dh_nll"])}


def _plain_clip(state):
    half = state["half"]
    small = torch.cat(state["grads"][:half]).float() if half else torch.zeros(0, device="cuda")
    large = torch.cat(state["grads"][half:])
    norm = (small.square().sum() + large.square().sum()).sqrt().view(1)
    coef = (state["max_norm"] / norm).clamp(max=1.0)
    return {"norm": norm, "coef": coef, "half": (small * coef).to(torch.bfloat16), "full": large * coef}


_RUN_PLAIN = {"decode": _plain_decode, "policy": _plain_policy, "pref": _plain_pref, "clip": _plain_clip}


def _workspace(n):
    return torch.empty(max(n, 256), device="cuda", dtype=torch.uint8)


def _call(state, build):
    """The descriptors of a call and its workspace: a program that calls again on the same buffers keeps them."""
    if "call" not in state:
        state["call"] = build(state)
    return state["call"]


def _build_decode(state):
    from paper_2606_19528_gb300 import lora
    projs = [lora.make_proj(lora.make_shape(state["T"], p["K"], p["N"], state["r"], state["scale"]), x=state["x"],
                            A=p.get("A"), B=p.get("B"), y=p["y"], Wq=lora.make_q4(p["codes"], p["params"]))
             for p in state["projs"]]
    projs = lora.make_projs(projs)
    ws = _workspace(lora.lora_decode_workspace_size(projs))
    return lora.lora_decode_q4, (projs, ws, ws.numel()), [p["y"] for p in state["projs"]]


def _build_policy(state):
    from paper_2606_19528_gb300 import lora
    kind = {"sum": lora.LORA_SUM, "tokens": lora.LORA_MEAN_TOKENS, "seqs": lora.LORA_MEAN_SEQS}[state["reduction"]]
    args = lora.make_policy_args(state["T"], state["seqs"], state["d"], state["offsets"], state["nll"],
                                 state["old_nll"], state["adv"], state["loss"],
                                 ref_nll=state["ref_nll"] if state["kl"] else None, mask=state["mask"],
                                 advantage_per_token=state["per_token"], clip_low=state["low"],
                                 clip_high=state["high"], beta=state["beta"], scale=state["scale"], reduction=kind,
                                 dh_nll=state["dh_nll"], dh=state["dh"], token_weight=state["token_weight"],
                                 stats=state["stats"])
    ws = _workspace(lora.lora_policy_workspace_size(args))
    return lora.lora_policy_fwd_bwd, (args, ws, ws.numel()), {k: state[k] for k in ("loss", "stats", "token_weight",
                                                                                   "dh")}


def _build_pref(state):
    from paper_2606_19528_gb300 import lora
    kind = {"sigmoid": lora.LORA_PREF_SIGMOID, "hinge": lora.LORA_PREF_HINGE,
            "square": lora.LORA_PREF_SQUARE}[state["kind"]]
    args = lora.make_pref_args(state["T"], state["seqs"] // 2, state["d"], state["offsets"], state["nll"],
                               state["loss"], ref_nll=state["ref_nll"] if state["ref"] else None, mask=state["mask"],
                               kind=kind, mean_tokens=state["mean_tokens"], beta=state["beta"],
                               margin=state["margin"], label_smoothing=state["smoothing"], scale=state["scale"],
                               dh_nll=state["dh_nll"], dh=state["dh"], token_weight=state["token_weight"],
                               rewards=state["rewards"])
    ws = _workspace(lora.lora_pref_workspace_size(args))
    return lora.lora_pref_fwd_bwd, (args, ws, ws.numel()), {k: state[k] for k in ("loss", "rewards", "token_weight",
                                                                                 "dh")}


def _build_clip(state):
    from paper_2606_19528_gb300 import lora
    half = state["half"]
    into = list(torch.split(state["packed"][0], [g.numel() for g in state["grads"][:half]])) if half else []
    into += list(torch.split(state["packed"][1], [g.numel() for g in state["grads"][half:]]))
    grads = lora.make_grads(list(zip(state["grads"], into)))
    ws = _workspace(lora.lora_clip_workspace_size(grads))
    out = {"norm": state["norm"], "coef": state["coef"], "half": state["packed"][0], "full": state["packed"][1]}
    return lora.lora_clip_grads, (grads, state["max_norm"], state["norm"], state["coef"], ws, ws.numel()), out


_BUILD = {"decode": _build_decode, "policy": _build_policy, "pref": _build_pref, "clip": _build_clip}


def _run_own(state):
    call, args, out = _call(state, _BUILD[state["op"]])
    call(*args)
    return out


_RUN_OWN = {op: _run_own for op in _BUILD}


# ---------------------------------------------------------------- work
def work(case):
    op = case["op"]
    if op == "decode":
        T, r, dims = case["T"], case["r"], _dims(case["dims"])
        by = 2 * T * dims[0][0] + sum(K * N // 2 + K * N // 16 + 2 * r * (K + N) + 2 * T * N for K, N in dims)
        return {"bytes": by, "flops": sum(2 * T * K * N + 2 * T * r * (K + N) for K, N in dims)}
    if op in ("policy", "pref"):
        T, d = case["T"], case["d"]
        trained = T * (1 - case["prompt"])
        per = (4 + 4 * case["kl"] + 4 * case["per_token"] if op == "policy" else 4 * case["ref"]) + 4
        return {"bytes": trained * (per + 2 * d) + T * (1 + 4 + 2 * d), "flops": trained * (d + 30)}
    sizes = [case["r"] * n for K, N in _dims(case["dims"]) for n in (K, N)] * case["layers"]
    half = min(case["half"], len(sizes) - 1)
    n16, n32 = sum(sizes[:half]), sum(sizes[half:])
    return {"bytes": 4 * n16 + 8 * n32, "flops": 3 * (n16 + n32)}


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"decode": _exact_decode, "policy": _exact_policy, "pref": _exact_pref, "clip": _exact_clip}[s["op"]](s)


def _exact_decode(s):
    x = s["x"].double()
    out = []
    for p in s["projs"]:
        y = torch.zeros(s["T"], p["N"], device="cuda", dtype=torch.float64)
        for n0 in range(0, p["N"], 8192):
            rows = slice(n0, min(p["N"], n0 + 8192))
            words = p["codes"][rows].contiguous().view(torch.int32).long()
            scale, offset = p["params"][rows].double().unbind(-1)
            scale, offset = (v.repeat_interleave(8, dim=1) for v in (scale, offset))
            for bit in range(0, 32, 4):  # column 8 m + 2 i (+ 1) of word m in bits 4 i (+ 16)
                col = 2 * (bit % 16 // 4) + bit // 16
                w = scale * ((words >> bit) & 15).double() + offset
                y[:, rows] += x[:, col::8] @ w.to(torch.bfloat16).double().T
        if s["r"]:
            for j in range(s["r"]):
                u = (x * p["A"][j].double()).sum(dim=1) * s["scale"]
                y += u[:, None] * p["B"][:, j].double()[None, :]
        out.append(y)
    return out


def _exact_policy(s):
    off = s["offsets"].tolist()
    on = s["mask"].bool()
    nll, old, ref, adv = (s[k].double() for k in ("nll", "old_nll", "ref_nll", "adv"))
    # whether a token is clipped goes by the 32-bit difference and the 32-bit logarithm of the bound
    d32 = s["old_nll"] - s["nll"]
    hi = torch.tensor(math.log1p(s["high"]), dtype=torch.float32).item()
    lo = torch.tensor(math.log1p(-s["low"]), dtype=torch.float32).item()
    loss, n_all = torch.zeros((), device="cuda", dtype=torch.float64), int(on.sum())
    kl_sum, clips = torch.zeros_like(loss), 0
    w = torch.zeros_like(nll)
    for i, (a, b) in enumerate(zip(off, off[1:])):
        t = torch.nonzero(on[a:b])[:, 0] + a
        if not t.numel():
            continue
        A = adv[t] if s["per_token"] else adv[i].expand(t.numel())
        rho = torch.exp(old[t] - nll[t])
        above, below = (A > 0) & (d32[t] > hi), (A < 0) & (d32[t] < lo)
        term = -A * rho
        term[above] = -A[above] * (1 + s["high"])
        term[below] = -A[below] * (1 - s["low"])
        slope = A * rho * ~(above | below)
        if s["kl"]:
            e = nll[t] - ref[t]
            kl = torch.exp(e) - 1 - e
            term = term + s["beta"] * kl
            slope = slope + s["beta"] * (torch.exp(e) - 1)
            kl_sum = kl_sum + kl.sum()
        norm = s["scale"] * {"sum": 1.0, "tokens": 1.0 / n_all, "seqs": 1.0 / (s["seqs"] * t.numel())}[s["reduction"]]
        loss = loss + norm * term.sum()
        w[t] = norm * slope
        clips += int((above | below).sum())
    stats = torch.stack([kl_sum / n_all, torch.tensor(clips / max(n_all, 1), device="cuda", dtype=torch.float64)])
    return {"loss": loss.view(1), "stats": stats, "token_weight": w, "dh": s["dh_nll"].double() * w[:, None]}


def _exact_pref(s):
    off = s["offsets"].tolist()
    on = s["mask"].bool()
    nll, ref, beta = s["nll"].double(), s["ref_nll"].double(), s["beta"]
    P = s["seqs"] // 2
    w, loss, rewards = torch.zeros_like(nll), 0.0, []
    for i in range(P):
        at = [torch.nonzero(on[off[j]:off[j + 1]])[:, 0] + off[j] for j in (2 * i, 2 * i + 1)]
        share = [1.0 / max(1, t.numel()) if s["mean_tokens"] else 1.0 for t in at]
        R = [c * float(((ref[t] if s["ref"] else 0.0) - nll[t]).sum()) for t, c in zip(at, share)]
        m = beta * (R[0] - R[1]) - s["margin"]
        if s["kind"] == "sigmoid":
            plus, minus = (math.log1p(math.exp(-abs(m))) + max(v, 0.0) for v in (m, -m))
            p = 1 / (1 + math.exp(-m)) if m > -700 else 0.0
            loss += (1 - s["smoothing"]) * minus + s["smoothing"] * plus
            slope = p - (1 - s["smoothing"])  # -(1 - e) (1 - p) + e p
        elif s["kind"] == "hinge":
            loss += max(0.0, 1 - m)
            slope = -1.0 if m < 1 else 0.0
        else:
            loss += (R[0] - R[1] - s["margin"] / beta - 0.5 / beta) ** 2
            slope = 2 * (R[0] - R[1] - s["margin"] / beta - 0.5 / beta) / beta
        w[at[0]] = -slope * beta * s["scale"] / P * share[0]
        w[at[1]] = slope * beta * s["scale"] / P * share[1]
        rewards += [beta * R[0], beta * R[1]]
    f = dict(device="cuda", dtype=torch.float64)
    return {"loss": torch.tensor([loss * s["scale"] / P], **f), "rewards": torch.tensor(rewards, **f),
            "token_weight": w, "dh": s["dh_nll"].double() * w[:, None]}


def _exact_clip(s):
    total = 0.0
    for g in s["grads"]:
        total += float(g.double().square().sum())
    norm = math.sqrt(total)
    coef = min(1.0, s["max_norm"] / norm) if norm else 1.0
    f = dict(device="cuda", dtype=torch.float64)
    half = s["half"]
    flat = [torch.cat([g.double() * coef for g in part]) if part else torch.zeros(0, **f)
            for part in (s["grads"][:half], s["grads"][half:])]
    return {"norm": torch.tensor([norm], **f), "coef": torch.tensor([coef], **f), "half": flat[0], "full": flat[1]}
