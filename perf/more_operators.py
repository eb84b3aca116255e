"""Operators around a recurrent ternary language model, as measurable cases: a
token mixer with a matrix state, beam search over the vocabulary with its
states, and distillation from a teacher.

``run`` computes an operator in its plain form, elementary torch operations,
or, where ``own`` is true, through the framework's entry points.  ``exact``
gives the same values in 64 bits.

Kinds of case:

  la       linear attention with a decay per head, from the stacked projection
           qkv [B*T][H (2 dk + dv)]: S_t = l S_{t-1} + k_t v_t^T, o_t = scale
           S_t^T q_t; o and the last state (updated in place for single tokens)
  la_bwd   its backward: the gradient of qkv in bfloat16, as the projection's
           own backward takes it, and of the first state
  beam     one step of beam search: the n best of W beams x V tokens from the
           beams' scores and logits, and (n = W) the recurrent states of all
           layers reordered after their parents in place
  distill  the divergence of a student's distribution over the vocabulary from
           a teacher's K best tokens; with its gradient, or ("grad" false)
           the loss alone
"""
import math

import torch

own = False

F32, F64, BF16, I32, U8 = torch.float32, torch.float64, torch.bfloat16, torch.int32, torch.uint8
INF = float("inf")


def listed():
    return [
        # One token of one sequence in generation (width 2048, 16 heads): the
        # state updated in place, pure latency.
        {"name": "la_token", "kind": "la", "B": 1, "T": 1, "H": 16, "dk": 128, "dv": 128, "f32": True, "s0": True},
        # One token of a running batch: bound by the states.
        {"name": "la_token_batch", "kind": "la", "B": 45, "T": 1, "H": 16, "dk": 128, "dv": 128, "f32": False,
         "s0": True},
        # Short ragged sequences, heads of odd widths, from a state.
        {"name": "la_ragged", "kind": "la", "B": 3, "T": 357, "H": 5, "dk": 80, "dv": 112, "f32": True, "s0": True},
        # A prompt of the paper's length at the 1.3B width, straight from the
        # projection's fp32 output.
        {"name": "la_prompt", "kind": "la", "B": 1, "T": 2048, "H": 16, "dk": 128, "dv": 128, "f32": True,
         "s0": False},
        # One long sequence in bfloat16.
        {"name": "la_long", "kind": "la", "B": 1, "T": 16384, "H": 16, "dk": 128, "dv": 128, "f32": False,
         "s0": True},
        # Training: short ragged sequences of a small model in bfloat16.
        {"name": "la_bwd_ragged", "kind": "la_bwd", "B": 3, "T": 357, "H": 8, "dk": 64, "dv": 64, "f32": False,
         "do_f32": False, "s0": True},
        # Training: four sequences of the paper's length at the 1.3B width.
        {"name": "la_bwd_train", "kind": "la_bwd", "B": 4, "T": 2048, "H": 16, "dk": 128, "dv": 128, "f32": True,
         "do_f32": True, "s0": False},
        # One request with four beams: 24 layers of MLGRU states.
        {"name": "beam_one", "kind": "beam", "B": 1, "W": 4, "V": 32000, "n": 4, "f32": True, "done": False,
         "first": False, "layers": 24, "row": 2048},
        # A few requests, twice as many candidates as beams (selection alone).
        {"name": "beam_wide", "kind": "beam", "B": 7, "W": 5, "V": 32001, "n": 10, "f32": False, "done": True,
         "first": False, "layers": 0, "row": 0},
        # A serving batch with matrix states (16 heads of 128 x 128).
        {"name": "beam_batch", "kind": "beam", "B": 32, "W": 8, "V": 50000, "n": 8, "f32": False, "done": True,
         "first": False, "layers": 2, "row": 262144},
        # The loss alone, over a few rows of a validation batch.
        {"name": "distill_eval", "kind": "distill", "M": 77, "V": 50001, "K": 20, "f32": True, "grad": False,
         "dz_f32": False, "tau": 1.0},
        # Training: the loss and the gradient of the logits over a batch.
        {"name": "distill_train", "kind": "distill", "M": 8192, "V": 32000, "K": 64, "f32": False, "grad": True,
         "dz_f32": False, "tau": 2.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the same ranges: sizes spread over their logarithms, head
    widths multiples of 16 (what the operator takes), everything else any."""
    kind = rng.choice(["la", "la", "la_bwd", "beam", "beam", "distill", "distill"])
    if kind in ("la", "la_bwd"):
        wide = rng.choice([64, 128, 128, 0])
        dk = wide or 16 * rng.randint(2, 8)
        dv = wide or 16 * rng.randint(2, 8)
        H = rng.choice([1, 3, 4, 8, 12, 16])
        B = rng.choice([1, 1, 2, 3, 4, 7])
        most = (8192 if kind == "la_bwd" else 16384) * 16 * 128 // (B * H * max(dk, dv))
        case = {"kind": kind, "B": B, "T": _log(rng, 33, min(16384, most)), "H": H, "dk": dk, "dv": dv,
                "f32": rng.random() < 0.5, "s0": rng.random() < 0.6}
        if kind == "la_bwd":
            case["do_f32"] = rng.random() < 0.5
        elif rng.random() < 0.4:
            case |= {"B": _log(rng, 1, 256), "T": rng.choice([1, 1, 1, 2, 4, 7]), "s0": True}
        return case
    if kind == "beam":
        B, W = _log(rng, 1, 32), rng.randint(2, 8)
        n = rng.choice([W, W, W, 2 * W, rng.randint(1, 16)])
        matrix = rng.random() < 0.4
        return {"kind": kind, "B": B, "W": W, "V": _log(rng, 1000, 50000), "n": n, "f32": rng.random() < 0.5,
                "done": rng.random() < 0.5, "first": rng.random() < 0.2,
                "layers": 0 if n != W else rng.randint(1, 2) if matrix else rng.randint(1, 24),
                "row": 0 if n != W else 16384 * rng.randint(1, 16) if matrix else 16 * rng.randint(16, 256)}
    f32 = rng.random() < 0.4
    V = _log(rng, 1000, 131072)
    return {"kind": kind, "M": _log(rng, 1, min(8192, 8192 * 16000 // V)), "V": V, "K": _log(rng, 1, 128), "f32": f32,
            "grad": rng.random() < 0.7, "dz_f32": rng.random() < 0.3, "tau": rng.choice([1.0, 2.0, 3.7])}


# ---------------------------------------------------------------------------
# inputs, from the seed alone
# ---------------------------------------------------------------------------

class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(240602528 + int(seed))

    def normal(self, *shape, scale=1.0, dtype=F32):
        t = torch.randn(shape, generator=self.g, device="cuda", dtype=F32)
        return t.mul_(scale).to(dtype) if scale != 1.0 else t.to(dtype)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=F32)


def _kind(f32):
    return F32 if f32 else BF16


def _empty(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _kept(st, bytes_of, *sizes):
    """The program's workspace, made at its first call and kept."""
    if "ws" not in st:
        st["ws"] = _empty(bytes_of(*sizes), dtype=U8)
    return st["ws"]


def _decay(H):
    """Decays from 1 - 2^-3 to 1 - 2^-11 over the heads, as models fix them."""
    h = torch.arange(H, device="cuda", dtype=F64) / max(1, H - 1)
    return (1.0 - 2.0 ** (-3.0 - 8.0 * h)).to(F32)


def prepare(case, seed):
    c, g = case, _Draw(seed)
    st = {"case": c}
    if c["kind"] in ("la", "la_bwd"):
        B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
        t = _kind(c["f32"])
        st |= {"qkv": g.normal(B * T, H * (2 * dk + dv), dtype=t), "decay": _decay(H),
               "s0": g.normal(B, H, dk, dv) if c["s0"] else None}
        if c["kind"] == "la":
            # single tokens go on from the state in place
            st |= {"o": _empty(B * T, H * dv, dtype=t),
                   "s_last": st["s0"] if T == 1 and c["s0"] else _empty(B, H, dk, dv)}
        else:
            st |= {"do": g.normal(B * T, H * dv, dtype=_kind(c["do_f32"])), "ds_last": g.normal(B, H, dk, dv),
                   "dqkv": _empty(B * T, H * (2 * dk + dv), dtype=BF16), "ds0": _empty(B, H, dk, dv)}
    elif c["kind"] == "beam":
        B, W, V, n = c["B"], c["W"], c["V"], c["n"]
        z = g.normal(B * W, V, scale=2.5)
        z[:, V // 2: V // 2 + 3] = -INF                      # tokens that the program bans
        scores = -30.0 * g.uniform(B, W)
        if c["first"]:
            scores = torch.full_like(scores, -INF)           # the first step: one beam holds the prompt
            scores[:, 0] = 0.0
        st |= {"logits": z.to(_kind(c["f32"])), "scores": scores, "end": 2,
               "done": (g.uniform(B, W) < 0.2).to(U8) if c["done"] else None,
               "new_scores": _empty(B, n), "tokens": _empty(B, n, dtype=I32), "parents": _empty(B, n, dtype=I32),
               "new_done": _empty(B, n, dtype=U8), "states": [g.normal(B * W, c["row"]) for _ in range(c["layers"])]}
    else:
        M, V, K = c["M"], c["V"], c["K"]
        z = g.normal(M, V, scale=2.0)
        # K tokens of each row, none twice; the teacher's logits fall off, and
        # the student has learnt a part of them
        at = (torch.randint(0, V, (M, 1), generator=g.g, device="cuda")
              + (V // K) * torch.arange(K, device="cuda")) % V
        t = 10.0 - 4.0 * torch.log1p(torch.arange(K, device="cuda", dtype=F32)) + g.normal(M, K)
        z.scatter_add_(1, at, 0.7 * t)
        valid = g.uniform(M, K) < 0.95
        valid[::17] = False                                  # rows of padding
        st |= {"z": z.to(_kind(c["f32"])), "idx": torch.where(valid, at, -1).to(I32), "t": t,
               "loss": _empty(M), "dloss": torch.full((M,), 1.0 / M, device="cuda"),
               "dz": _empty(M, V, dtype=_kind(c["dz_f32"])) if c["grad"] else None}
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _heads(x, B, T, H, w):
    """[B*T][H w] -> [B][H][T][w] in 32 bits."""
    return x.reshape(B, T, H, w).permute(0, 2, 1, 3).to(F32)


def _rows(x):
    """[B][H][T][w] -> [B*T][H w]."""
    B, H, T, w = x.shape
    return x.permute(0, 2, 1, 3).reshape(B * T, H * w)


def _split(st):
    c = st["case"]
    B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
    x = st["qkv"]
    return (_heads(x[:, :H * dk], B, T, H, dk), _heads(x[:, H * dk:2 * H * dk], B, T, H, dk),
            _heads(x[:, 2 * H * dk:], B, T, H, dv))


def _powers(decay, n):
    """decay[h] ** n, the power in 64 bits."""
    return decay.to(F64)[:, None].pow(n.to(F64).reshape(1, -1)).reshape(-1, *n.shape).to(F32)


def _attend(q, k, v, decay, E):
    """o_t = sum_{s <= t} l^(t - s) (q_t . k_s) v_s + l^t E^T q_t, in chunks
    whose states are joined by one product over the chunks."""
    B, H, T, _ = q.shape
    C = min(128, T)
    N = -(-T // C)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0, 0, N * C - T)).reshape(B, H, N, C, -1)  # noqa: E731
    q, k, v = cut(q), cut(k), cut(v)
    i, n = torch.arange(C, device="cuda"), torch.arange(N, device="cuda")
    low = i[:, None] - i[None, :]
    D = _powers(decay, low.clamp_min(0)) * (low >= 0)                    # [H][C][C]
    P = (q @ k.transpose(-1, -2)) * D[None, :, None]
    U = (k * _powers(decay, C - i)[None, :, None, :, None]).transpose(-1, -2) @ v   # [B][H][N][dk][dv]
    gap = n[:, None] - 1 - n[None, :]
    J = _powers(decay, C * gap.clamp_min(0)) * (gap >= 0)                # [H][N][N]
    S = (J[None] @ U.reshape(B, H, N, -1)).reshape(U.shape)
    if E is not None:
        S = S + _powers(decay, C * n)[None, :, :, None, None] * E[:, :, None]
    o = P @ v + _powers(decay, i)[None, :, None, :, None] * (q @ S)
    return o.reshape(B, H, N * C, -1)[:, :, :T]


def _last(k, v, decay, E, more):
    """sum_s l^(T - 1 - s + more) k_s v_s^T + l^(T - 1 + more) E."""
    T = k.shape[2]
    w = _powers(decay, T - 1 + more - torch.arange(T, device="cuda"))
    S = (k * w[None, :, :, None]).transpose(-1, -2) @ v
    return S if E is None else S + w[None, :, :1, None] * E


def _run_la(st):
    c = st["case"]
    B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
    scale = dk ** -0.5
    if own:
        import paper_2406_02528_amd as m
        m.mmf_linattn_fwd(st["qkv"], B, T, H, dk, dv, st["decay"], scale, st["s0"], st["o"], st["s_last"],
                          _kept(st, m.mmf_linattn_workspace_bytes, B, T, H, dk, dv))
        return {"o": st["o"], "s_last": st["s_last"]}
    q, k, v = _split(st)
    E = None if st["s0"] is None else st["s0"] * st["decay"][None, :, None, None]
    o = _rows(_attend(q, k, v, st["decay"], E) * scale).to(st["o"].dtype)
    st["s_last"].copy_(_last(k, v, st["decay"], E, 0))
    return {"o": o, "s_last": st["s_last"]}


def _run_la_bwd(st):
    c = st["case"]
    B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
    scale = dk ** -0.5
    if own:
        import paper_2406_02528_amd as m
        m.mmf_linattn_bwd(st["qkv"], B, T, H, dk, dv, st["decay"], scale, st["s0"], st["do"], st["ds_last"],
                          st["dqkv"], st["ds0"], _kept(st, m.mmf_linattn_bwd_workspace_bytes, B, T, H, dk, dv))
        return {"dqkv": st["dqkv"], "ds0": st["ds0"]}
    q, k, v = _split(st)
    do = _heads(st["do"], B, T, H, dv) * scale
    l, G = st["decay"], st["ds_last"]
    E = None if st["s0"] is None else (st["s0"] * l[None, :, None, None]).transpose(-1, -2)
    dq = _attend(do, v, k, l, E)
    q, k, v, do = (x.flip(2) for x in (q, k, v, do))
    dk_ = _attend(v, do, q, l, G.transpose(-1, -2)).flip(2)
    dv_ = _attend(k, q, do, l, G).flip(2)
    ds0 = _last(q, do, l, G, 1)
    return {"dqkv": torch.cat([_rows(dq), _rows(dk_), _rows(dv_)], 1).to(BF16), "ds0": ds0}


def _run_beam(st):
    c = st["case"]
    B, W, V, n = c["B"], c["W"], c["V"], c["n"]
    if own:
        import paper_2406_02528_amd as m
        m.mmf_beam_select(st["logits"], st["scores"], st["done"], st["end"], B, W, n, st["new_scores"], st["tokens"],
                          st["parents"], st["new_done"], _kept(st, m.mmf_beam_select_workspace_bytes, B, W, V, n))
        if st["states"]:
            m.mmf_beam_reorder(st["states"], st["parents"], B, W)
        return {"scores": st["new_scores"], "tokens": st["tokens"], "parents": st["parents"], "done": st["new_done"],
                "states": st["states"]}
    z = st["logits"].to(F32)
    if st["done"] is not None:
        over = st["done"].reshape(B * W, 1) != 0
        z = torch.where(over, -INF, z)
        z[:, st["end"]] = torch.where(over[:, 0], 0.0, z[:, st["end"]])
    z = torch.where(z.isnan(), -INF, z)
    # the n best of each row, then of all rows: scores next to each other are
    # told apart in 64 bits
    best, token = torch.sort(z, dim=1, descending=True, stable=True)
    best, token = best[:, :n].to(F64), token[:, :n]
    m_ = z.amax(1, keepdim=True).to(F64)
    lse = m_ + (z.to(F64) - m_).exp().sum(1, keepdim=True).log()
    score = (st["scores"].reshape(B * W, 1).to(F64) + (best - lse)).reshape(B, -1)
    top, at = torch.sort(score, dim=1, descending=True, stable=True)
    top, at = top[:, :n], at[:, :n]
    parents, tokens = at // best.shape[1], token.reshape(B, -1).gather(1, at)
    done = tokens == st["end"]
    if st["done"] is not None:
        done = done | (st["done"].gather(1, parents) != 0)
    if st["states"]:
        src = (parents + W * torch.arange(B, device="cuda")[:, None]).reshape(-1)
        [s.copy_(s[src]) for s in st["states"]]
    return {"scores": top.to(F32), "tokens": tokens.to(I32), "parents": parents.to(I32), "done": done.to(U8),
            "states": st["states"]}


def _run_distill(st):
    c = st["case"]
    tau = c["tau"]
    if own:
        import paper_2406_02528_amd as m
        if not c["grad"]:
            m.mmf_distill_fwd(st["z"], st["idx"], st["t"], tau, st["loss"])
            return {"loss": st["loss"]}
        m.mmf_distill_bwd(st["z"], st["idx"], st["t"], tau, st["dloss"], st["dz"], st["loss"])
        return {"loss": st["loss"], "dz": st["dz"]}
    z, idx = st["z"].to(F32), st["idx"].to(torch.int64)
    valid = idx >= 0
    some = valid.any(1, keepdim=True)
    x = z / tau
    m_ = x.amax(1, keepdim=True)
    e = (x - m_).exp()
    s = e.sum(1, keepdim=True)
    t = torch.where(valid, st["t"] / tau, -INF)
    t = torch.where(some, t, 0.0)
    u = (t - t.amax(1, keepdim=True)).to(F64)
    ln_p = u - u.exp().sum(1, keepdim=True).log()
    p = torch.where(valid, ln_p.exp(), 0.0)
    ln_q = (x.gather(1, idx.clamp_min(0)) - m_).to(F64) - s.to(F64).log()
    loss = tau * tau * torch.where(valid, p * (ln_p - ln_q), 0.0).sum(1)
    if not c["grad"]:
        return {"loss": loss.to(F32)}
    w = torch.where(some, st["dloss"][:, None] * tau, 0.0)
    dz = e * (w / s)
    dz.scatter_add_(1, idx.clamp_min(0), -(p * w).to(F32))
    return {"loss": loss.to(F32), "dz": dz.to(st["dz"].dtype)}


def run(state):
    return {"la": _run_la, "la_bwd": _run_la_bwd, "beam": _run_beam,
            "distill": _run_distill}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _tokens(x, B, T, H, w):
    """The rows of each token: T tensors [B][H][w] in 64 bits."""
    return x.reshape(B, T, H, w).to(F64).unbind(1)


def _exact_la(st):
    c = st["case"]
    B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
    l = st["decay"].to(F64)[None, :, None, None]
    q, k, v = (_tokens(x, B, T, H, w) for x, w in zip(st["qkv"].split([H * dk, H * dk, H * dv], 1), (dk, dk, dv)))
    S = torch.zeros(B, H, dk, dv, dtype=F64, device="cuda") if st["s0"] is None else st["s0"].to(F64)
    scale = dk ** -0.5
    if c["kind"] == "la":
        o = []
        for t in range(T):
            S = l * S + k[t][..., None] * v[t][..., None, :]
            o.append((q[t][..., None] * S).sum(2) * scale)
        return {"o": torch.stack(o, 1).reshape(B * T, H * dv), "s_last": S}
    do = _tokens(st["do"], B, T, H, dv)
    dq, dk_, dv_ = [], [None] * T, [None] * T
    for t in range(T):
        S = l * S + k[t][..., None] * v[t][..., None, :]
        dq.append((S * do[t][..., None, :]).sum(3) * scale)
    G = st["ds_last"].to(F64)
    for t in reversed(range(T)):
        G = G + scale * q[t][..., None] * do[t][..., None, :]
        dk_[t] = (G * v[t][..., None, :]).sum(3)
        dv_[t] = (G * k[t][..., None]).sum(2)
        G = l * G
    flat = lambda xs: torch.stack(xs, 1).reshape(B * T, -1)  # noqa: E731
    return {"dqkv": torch.cat([flat(dq), flat(dk_), flat(dv_)], 1), "ds0": G}


def _exact_beam(st):
    c = st["case"]
    B, W, V, n = c["B"], c["W"], c["V"], c["n"]
    lp = torch.log_softmax(st["logits"].to(F64).reshape(B, W, V), 2)
    if st["done"] is not None:
        alone = torch.full((V,), -INF, dtype=F64, device="cuda")
        alone[st["end"]] = 0.0
        lp[st["done"] != 0] = alone
    top, at = torch.topk((lp + st["scores"].to(F64)[..., None]).reshape(B, W * V), n, dim=1)
    states = [torch.stack([s.reshape(B, W, -1)[b, at[b] // V] for b in range(B)]).reshape(s.shape).to(F64)
              for s in st["states"]] if st["states"] and _small(st) else [None] * len(st["states"])
    return {"scores": top, "tokens": None, "parents": None, "done": None, "states": states}


def _small(st):
    return sum(s.numel() for s in st["states"]) < 1 << 24


def _exact_distill(st):
    c, tau = st["case"], st["case"]["tau"]
    M, V = c["M"], c["V"]
    z, idx = st["z"], st["idx"].to(torch.int64)
    loss, dz = torch.zeros(M, dtype=F64, device="cuda"), torch.zeros(M, V, dtype=F64, device="cuda") if c["grad"] else None
    for a in range(0, M, 512):  # some rows at a time: 64 bits of all would not fit
        r = slice(a, min(M, a + 512))
        lq = torch.log_softmax(z[r].to(F64) / tau, 1)
        ok = idx[r] >= 0
        lp = torch.log_softmax(torch.where(ok, st["t"][r].to(F64) / tau, -INF), 1)
        target = torch.zeros_like(lq)
        row = torch.arange(lq.shape[0], device="cuda")[:, None].expand_as(ok)[ok]
        target[row, idx[r][ok]] = lp[ok].exp()
        loss[r] = tau * tau * (torch.special.xlogy(target, target) - target * lq).sum(1)
        if c["grad"]:
            g = (lq.exp() - target) * (st["dloss"][r].to(F64) * tau)[:, None]
            dz[r] = torch.where(ok.any(1, keepdim=True), g, 0.0)
    return {"loss": loss, "dz": dz} if c["grad"] else {"loss": loss}


def exact(case, seed):
    st = prepare(case, seed)
    return {"la": _exact_la, "la_bwd": _exact_la, "beam": _exact_beam, "distill": _exact_distill}[case["kind"]](st)


def work(case):
    c = case
    size = lambda f32: 4 if f32 else 2  # noqa: E731
    if c["kind"] in ("la", "la_bwd"):
        B, T, H, dk, dv = c["B"], c["T"], c["H"], c["dk"], c["dv"]
        rows, wide, state = B * T * H, 2 * dk + dv, 4 * B * H * dk * dv
        if c["kind"] == "la":
            # each token joins the state (2 operations an entry) and reads it (2)
            return {"bytes": rows * (wide + dv) * size(c["f32"]) + state * (1 + c["s0"]), "flops": 4 * rows * dk * dv}
        # both states are followed and three products are read from them
        return {"bytes": rows * (wide * size(c["f32"]) + dv * size(c["do_f32"]) + 2 * wide) + state * (2 + c["s0"]),
                "flops": 10 * rows * dk * dv}
    if c["kind"] == "beam":
        B, W, V, n = c["B"], c["W"], c["V"], c["n"]
        return {"bytes": B * W * V * size(c["f32"]) + 13 * B * n + 5 * B * W + 8 * c["layers"] * B * W * c["row"],
                "flops": 4 * B * W * V}
    M, V, K = c["M"], c["V"], c["K"]
    return {"bytes": M * V * (size(c["f32"]) + (size(c["dz_f32"]) if c["grad"] else 0)) + M * (8 * K + 8),
            "flops": M * V * (8 if c["grad"] else 4)}
