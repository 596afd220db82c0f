"""Cases and calls shared by the tests of the linear attention, and the tolerances they are held to."""
from __future__ import annotations

import numpy as np

from oracle import linear

BF16_HALF_STEP = 2.0 ** -8
# Error of a sum of products beside the one final rounding, relative to the sum of the products' magnitudes:
#   weights of pairs, decayed sources and states enter products in two bf16 parts: 2^-17 each, a term meets two of them: 2^-16;
#   decays: sums of up to 64 log2 decays of at most 2^6 together, 7 additions rounded at 2^-24: 7 * 2^-18, a difference of two, times ln 2: under 2^-14.5
#     (where the sum is larger the weight is below 2^-64); passed on over N chunks of small sums: N * 2^-21, under 2^-15.5 for the 40 here;
#   fp32 accumulation: chains of at most 64 + 128 products and up to 40 rounds of the state: 2^-24 * 232, under 2^-16.
# Together under 2^-13.5.
TERMS = 2.0 ** -13


def bf16(x):
    """fp64 values of the array rounded to bf16."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().float().numpy().astype(np.float64)


def fp32(x):
    return np.asarray(x, dtype=np.float32).astype(np.float64)


class Case:
    """Rows and states in fp64, exactly representable in the types of the tensors."""

    def __init__(self, lengths, hq, hkv, d, seed=0, fixed=False, states=False, extra_rows=0, rate=0.1, scale=0.0):
        rng = np.random.default_rng(seed)
        self.lengths, self.hq, self.hkv, self.d, self.fixed = list(lengths), hq, hkv, d, fixed
        self.n, self.T = len(self.lengths), sum(self.lengths)
        self.rows = self.T + extra_rows
        self.scale, self.s = scale, scale or 1.0 / np.sqrt(np.float64(d))
        self.q, self.do = bf16(rng.standard_normal((self.rows, hq, d))), bf16(rng.standard_normal((self.rows, hq, d)))
        self.k, self.v = bf16(rng.standard_normal((self.rows, hkv, d))), bf16(rng.standard_normal((self.rows, hkv, d)))
        # every head its own rate, from ten times to a tenth of it
        per_head = rate * 10.0 ** rng.uniform(-1, 1, hkv)
        self.g = fp32(-per_head if fixed else -per_head * rng.exponential(1.0, (self.rows, hkv)))
        self.initial = fp32(3.0 * rng.standard_normal((self.n, hkv, d, d))) if states else None
        self.d_final = fp32(0.3 * rng.standard_normal((self.n, hkv, d, d))) if states else None
        self.cu = np.concatenate([[0], np.cumsum(self.lengths)]).astype(np.int64)

    def of_rows(self, x):
        return x[:self.T]

    @property
    def g_rows(self):
        return self.g if self.fixed else self.g[:self.T]

    def forward(self, absolute=False):
        f = np.abs if absolute else (lambda x: x)
        initial = None if self.initial is None else f(self.initial)
        return linear.forward(f(self.q[:self.T]), f(self.k[:self.T]), f(self.v[:self.T]), self.g_rows, self.lengths, self.s, initial)

    def backward(self, absolute=False):
        f = np.abs if absolute else (lambda x: x)
        opt = lambda x: None if x is None else f(x)
        out = linear.backward(f(self.q[:self.T]), f(self.k[:self.T]), f(self.v[:self.T]), self.g_rows, f(self.do[:self.T]), self.lengths, self.s,
                              opt(self.initial), opt(self.d_final))
        if self.fixed:
            out["dg"] = out["dg"].sum(0)
        return out

    # ---- on the GPU
    def to_device(self, fused=False, decay_stride=None):
        import torch
        cuda = lambda x, t=torch.bfloat16: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(t).cuda()
        self.tq, self.tk, self.tv, self.tdo = cuda(self.q), cuda(self.k), cuda(self.v), cuda(self.do)
        if fused:
            both = torch.cat([self.tq, self.tk, self.tv], dim=1).contiguous()
            self.tq, self.tk, self.tv = both[:, :self.hq], both[:, self.hq:self.hq + self.hkv], both[:, self.hq + self.hkv:]
        self.tg = cuda(self.g, torch.float32)
        if decay_stride is not None:
            wide = torch.full((self.rows, decay_stride), float("nan"), device="cuda")
            wide[:, :self.hkv] = self.tg
            self.tg = wide[:, :self.hkv]
        self.tcu = torch.from_numpy(self.cu).int().cuda()
        self.tinitial = None if self.initial is None else cuda(self.initial, torch.float32)
        self.td_final = None if self.d_final is None else cuda(self.d_final, torch.float32)
        return self

    def batch(self, A, hint=None, **slots):
        return A.LinearBatch(self.tcu, max_rows=max(self.lengths, default=0) if hint is None else hint, **slots)

    def run_forward(self, A, batch=None, final=True, stream=None, workspace=None):
        """(o, final states) as device tensors, NaN where nothing was written."""
        import torch
        batch = batch or self.batch(A)
        o = torch.full((self.rows, self.hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        out = torch.full((self.n, self.hkv, self.d, self.d), float("nan"), device="cuda") if final and self.n else None
        A.linear_attn_fwd(batch, self.tq, self.tk, self.tv, self.tg, o, self.workspace(A, batch, False) if workspace is None else workspace,
                          initial=self.tinitial, final=out, scale=self.scale, stream=stream)
        return o, out

    def workspace(self, A, batch, backward):
        import torch
        size = A.linear_attn_workspace_bytes(batch, self.rows, self.hq, self.hkv, self.d, backward=backward)
        return torch.full((size,), 255, dtype=torch.uint8, device="cuda")

    def run_backward(self, A, batch=None, f32=True, stream=None, workspace=None, decays=True):
        """dict of device tensors, NaN where nothing was written."""
        import torch
        batch = batch or self.batch(A)
        t = torch.float32 if f32 else torch.bfloat16
        nan = lambda shape, t=t: torch.full(shape, float("nan"), dtype=t, device="cuda")
        out = {"dq": nan((self.rows, self.hq, self.d)), "dk": nan((self.rows, self.hkv, self.d)), "dv": nan((self.rows, self.hkv, self.d))}
        if decays:
            out["dg"] = nan((self.hkv,) if self.fixed else (self.rows, self.hkv), torch.float32)
        if self.initial is not None:
            out["d_initial"] = nan((self.n, self.hkv, self.d, self.d), torch.float32)
        A.linear_attn_bwd(batch, self.tq, self.tk, self.tv, self.tg, self.tdo, out["dq"], out["dk"], out["dv"],
                          self.workspace(A, batch, True) if workspace is None else workspace, initial=self.tinitial, d_final=self.td_final,
                          d_log_decay=out.get("dg"), d_initial=out.get("d_initial"), scale=self.scale, stream=stream)
        return out


def host(x):
    return x.float().cpu().numpy().astype(np.float64)


def check(got, want, magnitude, half_step=2.0 ** -24, what=""):
    """Every element within one rounding of the result and TERMS of its terms."""
    got = host(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite at {np.argwhere(~np.isfinite(got))[:3].tolist()}"
    room = half_step * np.abs(want) + TERMS * magnitude + 1e-30
    off = np.abs(got - want)
    worst = np.unravel_index(np.argmax(off / room), off.shape) if off.size else ()
    assert not off.size or off[worst] <= room[worst], f"{what} at {worst}: {got[worst]} instead of {want[worst]}, {off[worst] / room[worst]:.2f} of what it may be off"


def check_forward(case, o, final=None):
    want, want_final = case.forward()
    most, most_final = case.forward(absolute=True)
    check(host(o)[:case.T], want, most, BF16_HALF_STEP, "o")
    assert np.isnan(host(o)[case.T:]).all(), "rows behind the last sequence were written"
    if final is not None:
        check(final, want_final, most_final, what="final state")


def check_backward(case, out, f32=True):
    want, most = case.backward(), case.backward(absolute=True)
    for name, x in out.items():
        rows = name in ("dq", "dk", "dv") or name == "dg" and not case.fixed
        got = host(x)
        if rows:
            assert np.isnan(got[case.T:]).all(), f"{name}: rows behind the last sequence were written"
            got = got[:case.T]
        magnitude = most[name]
        if name == "dg":
            # pairs across t come out of sums over a chunk's tokens and over its pairs: their terms are those of the chunk
            magnitude = chunk_magnitude(case, most)
        check(got, want[name], magnitude, BF16_HALF_STEP if not f32 and name in ("dq", "dk", "dv") else 2.0 ** -24, name)


def chunk_magnitude(case, most):
    """What a token's decay gradient is summed from: every pair of the segment's tokens that has one of them in its chunk, by the products' magnitudes."""
    q, k, dq, dk = np.abs(case.q[:case.T]), np.abs(case.k[:case.T]), most["dq"], most["dk"]
    G = case.hq // case.hkv
    per_row = (q * dq).sum(-1).reshape(case.T, case.hkv, G).sum(-1) + (k * dk).sum(-1)
    out = np.zeros((case.T, case.hkv))
    for a, e in zip(case.cu[:-1], case.cu[1:]):
        for c in range(a, e, 64):
            out[c:min(c + 64, e)] = per_row[c:min(c + 64, e)].sum(0)
        out[a:e] = np.maximum(out[a:e], out[a:e].max(0) if e > a else 0)
    out = out + most["dg"].reshape(-1, case.hkv).max(0) if not case.fixed else out
    return out.sum(0) if case.fixed else out
