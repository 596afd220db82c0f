"""Linear attention with a decay for each head, as a model that mixes such layers with softmax attention calls it, as cases that can
be timed and compared.

Three operators: the chunked form over packed sequences (`linear_attn_fwd`: training packs and prompts, states read and kept), its
gradients (`linear_attn_bwd`), and the recurrent form for one token per sequence over a pool of states (`linear_attn_step`).

Per sequence and KV head, with g the logarithm of a token's decay (g <= 0) and s the scale 1 / sqrt(head_dim):
  S_t = exp(g_t) S_{t-1} + k_t v_t^T,   o_t = s S_t^T q_t   for each query head of the group that shares the KV head.

A case is a dict of plain values:
  op         "fwd", "bwd", "step"
  heads, kv_heads, head_dim
  decay      "token": one decay per token and KV head; "head": one per KV head (a broadcast input)
  fused      q, k and v are views into one projection output
  fwd, bwd:  lengths (tokens of the packed sequences, separated by commas),
             states (fwd: initial states are read from a pool and final ones written to it; bwd: the gradient of the final states comes in and
             the one of the initial states goes out)
  bwd:       grads ("bf16" or "f32")
  step:      seqs
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _packed(name, op, lengths, heads, kv_heads, head_dim, decay="token", states=False, grads=None, fused=False):
    case = {"name": name, "op": op, "lengths": ",".join(str(n) for n in lengths), "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "decay": decay, "states": states, "fused": fused}
    return dict(case, grads=grads or "bf16") if op == "bwd" else case


def _step(name, seqs, heads, kv_heads, head_dim, decay="token", fused=False):
    return {"name": name, "op": "step", "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "decay": decay, "fused": fused}


# the repository's packs of mixed lengths: the smallest one, 16384 tokens with one long sequence, the headline pack
_TINY = (17, 64, 111)
_MIXED = (311, 627, 1059, 8192, 896, 2008, 846, 1128, 262, 1055)
_PACK = (1851, 8713, 1898, 4207, 450, 4813, 10836)


def listed():
    return [
        # the smallest pack: nothing but latency
        _packed("fwd_tiny", "fwd", _TINY, 2, 2, 64),
        # the headline pack on 24 heads: a training step's forward
        _packed("fwd_pack", "fwd", _PACK, 24, 24, 128),
        # further chunks of ten prompts of the width between the tile widths: states come out of the pool and go back
        _packed("fwd_prompts", "fwd", _MIXED, 16, 16, 104, states=True, fused=True),
        # one very long document on grouped heads with fixed decays: the work is along the tokens only
        _packed("fwd_long", "fwd", (131000,), 32, 8, 128, decay="head"),
        # gradients of the smallest pack
        _packed("bwd_tiny", "bwd", _TINY, 2, 2, 64),
        # the headline pack's backward
        _packed("bwd_pack", "bwd", _PACK, 24, 24, 128, fused=True),
        # one device's part of longer sequences, on grouped heads with learned fixed decays: gradients of states come in and go out
        _packed("bwd_grouped", "bwd", _MIXED, 32, 8, 128, decay="head", states=True),
        # equal sequences of a narrower head, fp32 gradients
        _packed("bwd_f32", "bwd", (2048,) * 4, 12, 12, 80, grads="f32"),
        # a single sequence's next token on a small share of the heads: the smallest call
        _step("step_one", 1, 5, 5, 128),
        # one generation step of 64 sequences on grouped heads
        _step("step_batch", 64, 32, 8, 128, fused=True),
        # of 500 sequences
        _step("step_many", 500, 16, 16, 104, decay="head"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# tokens x heads x columns of a drawn pack, and tokens x state elements; state elements of a drawn step: at most the largest listed ones'
_MOST_ELEMENTS = 1.0e8
_MOST_STATE_WORK = 1.2e10
_MOST_STATES = 8.0e7


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["fwd", "fwd", "bwd", "bwd", "step"])
    head_dim = rng.choice([128, 128, 128, 64, 104, 96, 80, 40, 32])
    while True:
        kv_heads = rng.randint(1, 8) if rng.random() < 0.5 else rng.choice([8, 12, 16, 24])
        heads = kv_heads * rng.choice([1, 1, 1, 2, 4, 5])
        decay, fused = rng.choice(["token", "token", "head"]), rng.random() < 0.5
        if op == "step":
            case = _step("", _log(rng, 1, 1024), heads, kv_heads, head_dim, decay, fused)
            fits = case["seqs"] * kv_heads * head_dim ** 2 <= _MOST_STATES
        else:
            seqs = _log(rng, 1, 64)
            lo = _log(rng, 1, 2000)
            hi = _log(rng, lo, 131072 if seqs == 1 else 16384)
            lengths = [_log(rng, lo, hi) for _ in range(seqs)]
            case = _packed("", op, lengths, heads, kv_heads, head_dim, decay, rng.random() < 0.4, rng.choice(["bf16", "bf16", "f32"]), fused)
            fits = sum(lengths) * heads * head_dim <= _MOST_ELEMENTS and sum(lengths) * heads * head_dim ** 2 <= _MOST_STATE_WORK
        if fits:
            del case["name"]
            return case


def _lengths(case):
    return [int(n) for n in case["lengths"].split(",")]


def work(case):
    """Every tensor read and written once; the products of the recurrent form."""
    hq, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    T = case["seqs"] if case["op"] == "step" else sum(_lengths(case))
    decays = 4 * hkv * (T if case["decay"] == "token" else 1)
    if case["op"] == "step":
        return {"bytes": 2 * T * d * (2 * hq + 2 * hkv) + decays + 2 * 4 * T * hkv * d * d, "flops": T * d * d * (3 * hkv + 2 * hq)}
    states = 2 * 4 * len(_lengths(case)) * hkv * d * d * case["states"]
    if case["op"] == "fwd":
        return {"bytes": 2 * T * d * (2 * hq + 2 * hkv) + decays + states, "flops": T * d * d * (3 * hkv + 2 * hq)}
    g = 4 if case["grads"] == "f32" else 2
    return {"bytes": 2 * T * d * (2 * hq + 2 * hkv) + g * T * d * (hq + 2 * hkv) + 2 * decays + states,
            "flops": T * d * d * (3 * hkv + 4 * hq + 5 * hkv)}


def prepare(case, seed):
    """Inputs on the device, output tensors, the workspace's size and the slots of the states."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    lengths = [1] * case["seqs"] if case["op"] == "step" else _lengths(case)
    T, B = sum(lengths), len(lengths)
    s = {"case": case, "max_rows": max(lengths)}
    if case["fused"]:
        both = randn(T, hq + 2 * hkv, d).bfloat16()
        s["q"], s["k"], s["v"] = both[:, :hq], both[:, hq:hq + hkv], both[:, hq + hkv:]
    else:
        s["q"], s["k"], s["v"] = (randn(T, h, d).bfloat16() for h in (hq, hkv, hkv))
    # heads that forget within a few tokens up to heads that remember some five hundred
    rate = 0.5 * 2.0 ** (-8.0 * (torch.arange(hkv, device="cuda") + torch.rand(hkv, generator=gen, device="cuda")) / hkv)
    s["log_decay"] = -rate if case["decay"] == "head" else -rate * torch.exp(0.5 * randn(T, hkv))
    ends = [0]
    for n in lengths:
        ends.append(ends[-1] + n)
    s["cu_rows"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    kept = case["op"] == "step" or case["states"]
    if case["op"] != "bwd":
        s["o"] = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
        if kept:
            slots = torch.randperm(B + 3, generator=gen, device="cuda")[:B].int()
            # what some tens of tokens leave in a state
            s["slots"], s["pool"] = slots, 4.0 * randn(B + 3, hkv, d, d)
            s["pool_out"] = torch.zeros(B + 3, hkv, d, d, device="cuda")
    else:
        s["d_o"] = randn(T, hq, d).bfloat16()
        t = torch.float32 if case["grads"] == "f32" else torch.bfloat16
        s["dq"], s["dk"], s["dv"] = (torch.empty(T, h, d, dtype=t, device="cuda") for h in (hq, hkv, hkv))
        s["d_log_decay"] = torch.empty_like(s["log_decay"])
        if kept:
            s["slots"], s["pool"] = torch.arange(B, device="cuda").int(), 4.0 * randn(B, hkv, d, d)
            s["d_final"], s["d_initial"] = 0.2 * randn(B, hkv, d, d), torch.empty(B, hkv, d, d, device="cuda")
    return s


def run(s):
    """One pass; the outputs are the state's own buffers where the framework writes them."""
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step}[op](s)


# ------------------------------------------------------------------------------------------- the framework's calls
def _own(s, op):
    import paper_2504_20490_amd as A
    slots = s.get("slots")
    if op == "step":
        batch = A.LinearBatch(None, initial_slots=slots, final_slots=slots)
        A.linear_attn_step(batch, s["q"], s["k"], s["v"], s["log_decay"], s["o"], initial=s["pool"], final=s["pool_out"])
        return {"o": s["o"], "states": s["pool_out"]}
    batch = A.LinearBatch(s["cu_rows"], max_rows=s["max_rows"], initial_slots=slots, final_slots=slots)
    T, hq, d = s["q"].shape
    if "ws" not in s:
        size = A.linear_attn_workspace_bytes(batch, T, hq, s["k"].shape[1], d, backward=op == "bwd")
        s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    if op == "fwd":
        A.linear_attn_fwd(batch, s["q"], s["k"], s["v"], s["log_decay"], s["o"], s["ws"], initial=s.get("pool"), final=s.get("pool_out"))
        return {"o": s["o"], "states": s["pool_out"]} if "pool" in s else {"o": s["o"]}
    A.linear_attn_bwd(batch, s["q"], s["k"], s["v"], s["log_decay"], s["d_o"], s["dq"], s["dk"], s["dv"], s["ws"], initial=s.get("pool"),
                      d_final=s.get("d_final"), d_log_decay=s["d_log_decay"], d_initial=s.get("d_initial"))
    return {name: s[name] for name in ("dq", "dk", "dv", "d_log_decay", "d_initial") if name in s}


# ------------------------------------------------------------------------------------------- the plain forms
_CHUNK = 128


class _Chunks:
    """The packed tokens cut into chunks; places x of `rows` that lie behind their sequence's end are not `real`.  Sequence s takes
    the chunks from cu[s] // _CHUNK + s on, which leaves room for all of its own."""

    def __init__(self, s):
        cu = s["cu_rows"].long()
        T, B = s["q"].shape[0], cu.shape[0] - 1
        self.tokens = T
        first = cu[:-1] // _CHUNK + torch.arange(B, device="cuda")
        x = torch.arange(T // _CHUNK + B, device="cuda")
        self.seq = torch.searchsorted(first, x, right=True) - 1
        rows = (cu[self.seq] + (x - first[self.seq]) * _CHUNK)[:, None] + torch.arange(_CHUNK, device="cuda")
        self.real = rows < cu[self.seq + 1][:, None]                                     # [X, C]
        self.rows, self.put = rows.clamp(max=T - 1), torch.where(self.real, rows, T)     # (what is not real is put behind the last row)
        g = s["log_decay"].expand(T, -1).double()[self.rows] * self.real[..., None]
        self.G = g.cumsum(1).transpose(1, 2)                                             # [X, H, C], in 64 bits as everything along the tokens
        C = self.G[..., -1].cumsum(0).T                                                  # [H, X]: up to and with a chunk
        before = C - self.G[..., -1].T
        same = self.seq[:, None] == self.seq
        later = x[:, None] > x
        # what is left of chunk y's state at the start of chunk x, and of the state at a sequence's start; likewise at its end
        self.to_later = torch.exp(before[:, :, None] - C[:, None, :]).masked_fill(~(same & later), 0.0).nan_to_num(posinf=0.0).float()
        self.from_start = torch.exp(before - before[:, first[self.seq]]).float()
        end = C[:, torch.cat([first[1:], first.new_tensor([len(x)])]) - 1]               # [H, B]
        self.to_end = torch.exp((end[:, self.seq] - C)).float()                          # [H, X]
        self.whole = torch.exp(end - before[:, first]).float()                           # [H, B]
        self.of_seq = (self.seq == torch.arange(B, device="cuda")[:, None]).float()      # [B, X]
        i = torch.arange(_CHUNK, device="cuda")
        self.D = torch.exp(self.G[..., :, None] - self.G[..., None, :]).masked_fill(i[:, None] < i, 0.0).nan_to_num(posinf=0.0).float()
        self.inward = torch.exp(self.G).float()                                          # a chunk's start to token i
        self.outward = torch.exp(self.G[..., -1:] - self.G).float()                      # token j to the chunk's end

    def cut(self, x, groups=1):
        """[T, H * groups, d] as fp32 [X, H, groups * C, d], zero where there is no token."""
        y = x[self.rows].float() * self.real[..., None, None]
        X, C, h, d = y.shape
        return y.view(X, C, h // groups, groups, d).permute(0, 2, 3, 1, 4).reshape(X, h // groups, groups * C, d)

    def joined(self, y, like):
        """The inverse of cut, in the type of `like`."""
        X, H, n, d = y.shape
        y = y.view(X, H, n // _CHUNK, _CHUNK, d).permute(0, 3, 1, 2, 4).reshape(X, _CHUNK, -1, d)
        return self.in_rows(y.to(like.dtype))

    def in_rows(self, y):
        out = torch.empty(self.tokens + 1, *y.shape[2:], dtype=y.dtype, device="cuda")
        out[self.put] = y
        return out[:-1]

    def at_starts(self, U, initial):
        """The states at the chunks' starts from what each chunk adds, [X, H, d, d]."""
        X, H, d, _ = U.shape
        S = torch.bmm(self.to_later, U.transpose(0, 1).reshape(H, X, d * d)).view(H, X, d, d).transpose(0, 1)
        return S if initial is None else S + self.from_start.T[..., None, None] * initial[self.seq]

    def at_ends(self, dU, final):
        """The same in the other direction: what reaches the chunks' ends from the later ones."""
        X, H, d, _ = dU.shape
        R = torch.bmm(self.to_later.transpose(1, 2).contiguous(), dU.transpose(0, 1).reshape(H, X, d * d)).view(H, X, d, d).transpose(0, 1)
        return R if final is None else R + self.to_end.T[..., None, None] * final[self.seq]


def _times(x, w, groups):
    """x [X, H, groups * C, d] times w [X, H, C] along the tokens."""
    return x * w.repeat(1, 1, groups)[..., None]


def _plain_fwd(s):
    G, scale = s["q"].shape[1] // s["k"].shape[1], s["q"].shape[2] ** -0.5
    c = _Chunks(s)
    q, k, v = c.cut(s["q"], G) * scale, c.cut(s["k"]), c.cut(s["v"])
    initial = s["pool"][s["slots"].long()] if "pool" in s else None
    U = (_times(k, c.outward, 1)).transpose(2, 3) @ v
    S = c.at_starts(U, initial)
    P = (q @ k.transpose(2, 3)) * c.D.repeat(1, 1, G, 1)
    out = {"o": c.joined(P @ v + _times(q @ S, c.inward, G), s["o"])}
    if initial is None:
        return out
    X, H, d, _ = U.shape
    final = torch.bmm(c.of_seq * c.to_end[:, None, :], U.transpose(0, 1).reshape(H, X, d * d)).view(H, -1, d, d).transpose(0, 1)
    s["pool_out"][s["slots"].long()] = final + c.whole.T[..., None, None] * initial
    return dict(out, states=s["pool_out"])


def _plain_bwd(s):
    G, scale = s["q"].shape[1] // s["k"].shape[1], s["q"].shape[2] ** -0.5
    c = _Chunks(s)
    q, do, k, v = c.cut(s["q"], G) * scale, c.cut(s["d_o"], G), c.cut(s["k"]), c.cut(s["v"])
    initial, d_final = s.get("pool"), s.get("d_final")
    S = c.at_starts(_times(k, c.outward, 1).transpose(2, 3) @ v, initial)
    dU = _times(q, c.inward, G).transpose(2, 3) @ do
    R = c.at_ends(dU, d_final)
    D = c.D.repeat(1, 1, G, 1)
    QK, DV = (q @ k.transpose(2, 3)) * D, (do @ v.transpose(2, 3)) * D
    dq_far, dk_far = _times(do @ S.transpose(2, 3), c.inward, G), _times(v @ R.transpose(2, 3), c.outward, 1)
    dq = DV @ k + dq_far
    dk = DV.transpose(2, 3) @ q + dk_far
    dv = QK.transpose(2, 3) @ do + _times(k @ R, c.outward, 1)
    # d g_t: the pairs of a later and an earlier token that t lies between, by where the two are
    X, H, n, _ = q.shape
    i = torch.arange(_CHUNK, device="cuda")
    W = (QK * (do @ v.transpose(2, 3))).view(X, H, G, _CHUNK, _CHUNK).sum(2).masked_fill(i[:, None] <= i, 0.0)
    a = (q * dq_far).sum(-1).view(X, H, G, _CHUNK).sum(2)
    b = (k * dk_far).sum(-1)
    from_here = lambda x: x.flip(-1).double().cumsum(-1).flip(-1)
    across = c.inward[..., -1].double() * (S * R).sum((2, 3), dtype=torch.float64)
    dg = from_here(W.sum(3) - W.sum(2)) + from_here(a) + (b.double().cumsum(-1) - b) + across[..., None]
    dg = c.in_rows(dg.transpose(1, 2))                                                   # [T, H]
    # (q carries the scale: dq is to lose it once more)
    out = {"dq": c.joined(dq * scale, s["dq"]), "dk": c.joined(dk, s["dk"]), "dv": c.joined(dv, s["dv"]),
           "d_log_decay": (dg if s["case"]["decay"] == "token" else dg.sum(0)).float()}
    if initial is None:
        return out
    X, H, d, _ = dU.shape
    d_initial = torch.bmm(c.of_seq * c.from_start[:, None, :], dU.transpose(0, 1).reshape(H, X, d * d)).view(H, -1, d, d).transpose(0, 1)
    return dict(out, d_initial=d_initial + c.whole.T[..., None, None] * d_final)


def _plain_step(s):
    B, hq, d = s["q"].shape
    hkv = s["k"].shape[1]
    slots = s["slots"].long()
    S = s["pool"][slots] * torch.exp(s["log_decay"].expand(B, -1))[..., None, None] + s["k"].float()[..., None] * s["v"].float()[:, :, None]
    s["pool_out"][slots] = S
    o = s["q"].float().view(B, hkv, hq // hkv, d) @ S * d ** -0.5
    return {"o": o.view(B, hq, d).bfloat16(), "states": s["pool_out"]}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
_BLOCK = 32


def exact(case, seed):
    """The recurrence, _BLOCK tokens at a time: S_t = e^(G_t) S_0 + sum_j e^(G_t - G_j) k_j v_j^T with G the sum of g from the block's start."""
    s = prepare(case, seed)
    f64, hq, hkv, d = torch.float64, case["heads"], case["kv_heads"], case["head_dim"]
    scale, group = 1.0 / math.sqrt(d), hq // hkv
    T = s["q"].shape[0]
    g = s["log_decay"].to(f64).expand(T, hkv)
    per_head = lambda x: x.to(f64).movedim(0, 1)                                           # [heads, tokens, d]
    q, k, v = per_head(s["q"]), per_head(s["k"]), per_head(s["v"])
    if case["op"] == "step":
        slots = s["slots"].long()
        states = s["pool_out"].to(f64)
        states[slots] = torch.exp(g)[:, :, None, None] * s["pool"].to(f64)[slots] + torch.einsum("hta,htb->thab", k, v)
        heads = torch.arange(hq, device="cuda") // group
        return {"o": scale * torch.einsum("hta,thab->thb", q, states[slots][:, heads]), "states": states}
    wide = lambda x: x.repeat_interleave(group, 0)                                         # KV heads to query heads
    narrow = lambda x: x.unflatten(0, (hkv, group)).sum(1)
    out = {name: [] for name in (("o",) if case["op"] == "fwd" else ("dq", "dk", "dv", "d_log_decay"))}
    states = s["pool_out"].to(f64) if "pool_out" in s else None
    d_initial = []
    start = 0
    for n_seq, length in enumerate(_lengths(case)):
        S = s["pool"][s["slots"][n_seq].long()].to(f64) if "pool" in s else torch.zeros(hkv, d, d, dtype=f64, device="cuda")
        blocks = [(a, min(a + _BLOCK, start + length)) for a in range(start, start + length, _BLOCK)]
        piece = {name: [] for name in out}
        for a, e in blocks:                                                                # forwards: S at each block's start
            G = g[a:e].cumsum(0).T                                                         # [hkv, n]
            gap = G[:, :, None] - G[:, None, :]
            keep = torch.exp(gap.tril()) * torch.ones_like(gap).tril()
            read, kb, vb = (q if case["op"] == "fwd" else per_head(s["d_o"][a:e])), k[:, a:e], v[:, a:e]
            if case["op"] == "fwd":
                x = read[:, a:e]
                o = wide(torch.exp(G))[..., None] * (x @ wide(S)) + (wide(keep) * (x @ wide(kb).mT)) @ wide(vb)
                piece["o"].append(scale * o)
            else:
                o = wide(torch.exp(G))[..., None] * (read @ wide(S).mT) + (wide(keep) * (read @ wide(vb).mT)) @ wide(kb)
                piece["dq"].append(scale * o)
            left = torch.exp(G[:, -1:] - G)[..., None]
            S = torch.exp(G[:, -1])[:, None, None] * S + (left * kb).mT @ vb
        if case["op"] == "fwd":
            if states is not None:
                states[s["slots"][n_seq].long()] = S
        else:
            R = s["d_final"][n_seq].to(f64) if "d_final" in s else torch.zeros_like(S)
            last = (S * R).sum((1, 2))                                                     # <S, dS> behind the last token
            for a, e in reversed(blocks):
                G = g[a:e].cumsum(0).T
                gap = G[:, :, None] - G[:, None, :]
                keep = wide(torch.exp(gap.tril()) * torch.ones_like(gap).tril())
                qb, kb, vb, db = scale * q[:, a:e], k[:, a:e], v[:, a:e], per_head(s["d_o"][a:e])
                left = torch.exp(G[:, -1:] - G)[..., None]
                piece["dk"].insert(0, left * (vb @ R.mT) + narrow((keep * (db @ wide(vb).mT)).mT @ qb))
                piece["dv"].insert(0, left * (kb @ R) + narrow((keep * (qb @ wide(kb).mT)).mT @ db))
                R = torch.exp(G[:, -1])[:, None, None] * R + narrow((wide(torch.exp(G))[..., None] * qb).mT @ db)
            d_initial.append(R)
            # e^(g_t) <S_(t-1), dS_t> = <S_last, dS_last> + the sum over the tokens from t on of <q, dq> - <k, dk>
            at = slice(start, start + length)
            net = narrow((q[:, at] * torch.cat(piece["dq"], 1)).sum(-1)) - (k[:, at] * torch.cat(piece["dk"], 1)).sum(-1)
            piece["d_log_decay"] = [(last[:, None] + net.flip(1).cumsum(1).flip(1))]
        for name in out:
            out[name].append(torch.cat(piece[name], 1).movedim(0, 1))
        start += length
    out = {name: torch.cat(x) for name, x in out.items()}
    if case["op"] == "fwd":
        return out if states is None else dict(out, states=states)
    if case["decay"] == "head":
        out["d_log_decay"] = out["d_log_decay"].sum(0)
    return dict(out, d_initial=torch.stack(d_initial)) if "d_final" in s else out
