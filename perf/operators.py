"""What a generation or evaluation program has the library do around a paged key/value cache, as cases that can be timed and compared.

Four operators: rotary embedding with positions on several axes (`rope_axes_qk`, also turned back for gradients), the write of
new tokens into the cache with the rotation and the quantisation fused in (`kv_cache_write`), the read of cached tokens back into
packed bf16 tensors (`kv_cache_read`), and the attention of new tokens over the cache (`attn_paged_fwd`: prompt chunks, several
tokens, single tokens, mixed).

A case is a dict of plain values:
  op         "axes", "write", "read", "attn"
  heads, kv_heads, head_dim
  axes:  tokens, num_axes (1 to 3), grads ("bf16" or "f32"), inverse, fused (q and k are views into one projection output),
         grid (tokens of a picture's row and column: the positions walk through time, height and width)
  the others: cache ("bf16" or "e4m3"), page_size, seqs, rows_lo / rows_hi (new tokens of a sequence, drawn evenly over their logarithm),
         chunks (this many of the sequences bring chunk_rows new tokens instead), past_lo / past_hi (tokens cached before them, likewise),
         pack (the seed of the lengths: the same pack for every seed of the values)
  write: rotate (False: k and v are written as they are)

Conventions of the cache: pages [num_pages, kv_heads, page_size, row], row = head_dim (bf16) or head_dim rounded up to 16 (e4m3, the
rest zero); e4m3 rows stand for value * 2^(scale - 127) with one scale byte per token and head, the smallest power of two from 2^-100 on
that keeps the row's largest magnitude at 448 or below.  Row r of a sequence that brings n rows sits at position kv_len - n + r.
"""
from __future__ import annotations

import math
import random

import torch

own = False

ROPE_BASE = 10000.0


def _axes(name, tokens, heads, kv_heads, head_dim, num_axes=3, grads="bf16", inverse=False, fused=False, grid=24):
    return {"name": name, "op": "axes", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "num_axes": num_axes, "grads": grads, "inverse": inverse, "fused": fused, "grid": grid}


def _paged(name, op, heads, kv_heads, head_dim, cache, seqs, rows, past, page_size=16, pack=1, chunks=0, chunk_rows=1, rotate=True):
    case = {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "cache": cache, "seqs": seqs,
            "rows_lo": rows[0], "rows_hi": rows[1], "past_lo": past[0], "past_hi": past[1], "chunks": chunks,
            "chunk_rows": chunk_rows, "page_size": page_size, "pack": pack}
    return dict(case, rotate=rotate) if op == "write" else case


def listed():
    return [
        # the repository's smallest pack with picture positions: nothing but latency
        _axes("axes_tiny", 192, 2, 2, 64, grid=8),
        # the headline pack's tokens on 24 heads, as the frames of a video; q and k views into one projection output
        _axes("axes_video", 32768, 24, 24, 128, fused=True, grid=24),
        # the gradients of a layer on grouped KV heads, turned back in fp32
        _axes("axes_grads", 16384, 32, 8, 128, grads="f32", inverse=True, grid=32),
        # one generation step of 64 sequences: rotate, quantise, write
        _paged("write_step", "write", 32, 8, 128, "e4m3", 64, (1, 1), (100, 4000), 16, 2),
        # prompts of the width that lies between the tile widths, into a bf16 cache
        _paged("write_prompts", "write", 16, 16, 104, "bf16", 10, (262, 8192), (0, 0), 64, 3),
        # short prefixes of a small share of the heads, read back
        _paged("read_tiny", "read", 2, 2, 64, "bf16", 3, (17, 111), (0, 40), 16, 4),
        # long prefixes out of the 8-bit cache: the packed tensors that a training step recomputes on
        _paged("read_prefixes", "read", 32, 8, 128, "e4m3", 14, (315, 29082), (0, 0), 64, 5),
        # a single sequence's next token on a small share of the heads: the smallest attention
        _paged("decode_one", "attn", 5, 5, 128, "bf16", 1, (1, 1), (1057, 1057), 16, 6),
        # one generation step of 64 sequences over the 8-bit cache
        _paged("decode_batch", "attn", 32, 8, 128, "e4m3", 64, (1, 1), (500, 16000), 16, 7),
        # one token over a very long document: the work is along the keys only
        _paged("decode_long", "attn", 32, 8, 128, "bf16", 1, (1, 1), (131000, 131000), 64, 8),
        # a prompt's chunk behind a long prefix
        _paged("chunk_long", "attn", 32, 8, 128, "bf16", 1, (2048, 2048), (27034, 27034), 64, 9),
        # chunks and single tokens in one call, 8-bit cache, the width between the tile widths
        _paged("mixed", "attn", 16, 16, 104, "e4m3", 26, (1, 1), (200, 8000), 16, 10, chunks=2, chunk_rows=700),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# pairs of (padded) rows and keys x query heads of a drawn attention, and elements of a drawn copy: below the largest listed ones
_MOST_PAIRS = 1.6e9
_MOST_ELEMENTS = 1.3e8


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["axes", "axes", "write", "write", "read", "attn", "attn", "attn", "attn"])
    head_dim = rng.choice([128, 128, 128, 64, 104, 96, 80, 40])
    kv_heads = rng.randint(1, 8) if rng.random() < 0.5 else rng.choice([8, 12, 16, 24])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 5, 8])
    while True:
        if op == "axes":
            case = _axes("", _log(rng, 1, 65536), heads, kv_heads, head_dim, rng.choice([1, 2, 3, 3]), rng.choice(["bf16", "f32"]),
                         rng.random() < 0.5, rng.random() < 0.5, rng.randint(4, 40))
            fits = case["tokens"] * (heads + kv_heads) * head_dim <= _MOST_ELEMENTS
        else:
            seqs, most = _log(rng, 1, 96), 1 if op == "attn" else 2000
            rows = (1, 1) if op != "read" and rng.random() < 0.5 else (1, _log(rng, 2, 8 * most + 16))
            chunks = rng.randint(1, min(seqs, 3)) if op == "attn" and rng.random() < 0.4 else 0
            case = _paged("", op, heads, kv_heads, head_dim, rng.choice(["bf16", "e4m3"]), seqs, rows,
                          (_log(rng, 1, 500), _log(rng, 500, 131072 if seqs < 3 else 16384)), rng.choice([16, 32, 64, 256]),
                          rng.randrange(1 << 20), chunks, _log(rng, 16, 2048) if chunks else 1, rng.random() < 0.7)
            rows, lens = _geometry(case)
            padded = max(rows) * max(lens) * seqs * heads
            fits = (sum(lens) * kv_heads * head_dim <= _MOST_ELEMENTS * 2 and sum(rows) * heads * head_dim <= _MOST_ELEMENTS
                    and (op != "attn" or (padded <= _MOST_PAIRS and seqs * max(lens) * kv_heads * head_dim <= 8 * _MOST_ELEMENTS)))
        if fits:
            del case["name"]
            return case


def _geometry(case):
    """(new tokens, tokens in the cache with them) of every sequence."""
    rng = random.Random(case["pack"])
    rows = [case["chunk_rows"] if s < case["chunks"] else _log(rng, case["rows_lo"], case["rows_hi"]) for s in range(case["seqs"])]
    past = [_log(rng, max(case["past_lo"], 1), case["past_hi"]) if case["past_hi"] else 0 for s in range(case["seqs"])]
    order = sorted(range(case["seqs"]), key=lambda s: rng.random())
    return [rows[s] for s in order], [rows[s] + past[s] for s in order]


def _row(case):
    d = case["head_dim"]
    return d if case["cache"] == "bf16" else (d + 15) // 16 * 16


def work(case):
    """Every tensor read and written once; the products over the visible pairs."""
    hq, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "axes":
        T, g = case["tokens"], 4 if case["grads"] == "f32" else 2
        distinct = min(T, max(T // case["grid"] ** 2, case["grid"]) + 1)
        return {"bytes": 2 * g * T * (hq + hkv) * d + 4 * T * case["num_axes"] + 4 * d * distinct, "flops": 3 * T * (hq + hkv) * d}
    rows, lens = _geometry(case)
    T, keys = sum(rows), sum(lens)
    cached = hkv * (2 * d if case["cache"] == "bf16" else d + 1)       # bytes of a token's k, or v
    if case["op"] == "write":
        turned = 2 * 2 * T * hq * d + 4 * d * T if case["rotate"] else 0
        return {"bytes": 2 * T * (2 * hkv * d + cached) + turned, "flops": T * d * (3 * (hq + hkv) * case["rotate"] + 2 * hkv)}
    if case["op"] == "read":
        return {"bytes": 2 * T * (2 * hkv * d + cached), "flops": 2 * T * hkv * d}
    pairs = sum(n * (kv - n) + n * (n + 1) // 2 for n, kv in zip(rows, lens))
    return {"bytes": 2 * keys * cached + 2 * 2 * T * hq * d + 4 * T * hq, "flops": 4 * d * pairs * hq}


def _table(positions, d):
    theta = ROPE_BASE ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * theta
    return torch.stack([a.cos(), a.sin()], dim=-1).float().contiguous()


def _pair_axis(num_axes, half):
    """The pairs' axes in sections: time takes the first, height and width share the rest."""
    edges = {1: [half], 2: [half // 2, half], 3: [half // 4, half // 4 + (half - half // 4) // 2, half]}[num_axes]
    return [sum(i >= e for e in edges) for i in range(half)]


def _randn(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def prepare(case, seed):
    """Inputs on the device, output tensors, the workspace, and the pool with its page table."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    s = {"case": case, "heads": hq}
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    if case["op"] == "axes":
        T, dtype = case["tokens"], torch.float32 if case["grads"] == "f32" else torch.bfloat16
        if case["fused"]:
            both = _randn(gen, T, hq + hkv, d, dtype=dtype)
            s["q"], s["k"] = both[:, :hq], both[:, hq:]
        else:
            s["q"], s["k"] = _randn(gen, T, hq, d, dtype=dtype), _randn(gen, T, hkv, d, dtype=dtype)
        s["q_out"], s["k_out"] = (torch.empty(T, h, d, dtype=dtype, device="cuda") for h in (hq, hkv))
        # pictures of grid x grid tokens, one after the other; the first token's place by the seed
        t = torch.arange(T, device="cuda") + seed % 1000
        g = case["grid"]
        s["positions"] = torch.stack([t // (g * g), t // g % g, t % g][:case["num_axes"]] if case["num_axes"] > 1 else [t]).int()
        s["table_positions"] = int(s["positions"].max()) + 1
        s["table"] = _table(s["table_positions"], d)
        s["pair_axis"] = _pair_axis(case["num_axes"], d // 2)
        return s
    rows, lens = _geometry(case)
    T, size, width = sum(rows), case["page_size"], _row(case)
    pages = [-(-n // size) for n in lens]
    num_pages = sum(pages) + 3
    ends = [0]
    for n in rows:
        ends.append(ends[-1] + n)
    s.update(cu_rows=ints(ends), kv_lens=ints(lens), max_rows=max(rows))
    order = torch.randperm(num_pages, generator=gen, device="cuda").int()
    table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    s["page_table"] = table
    shape = (num_pages, hkv, size, width)
    if case["cache"] == "bf16":
        s["k_cache"], s["v_cache"] = _randn(gen, *shape), _randn(gen, *shape)
        s["k_scale"] = s["v_scale"] = None
    else:
        # rows of values around one whose largest magnitude, some three, lies between 224 and 448 in units of the scale
        for x in "kv":
            s[x + "_cache"] = _randn(gen, *shape, dtype=torch.float32).mul_(110.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
            s[x + "_cache"][..., d:] = 0
            s[x + "_scale"] = torch.randint(119, 122, shape[:3], generator=gen, device="cuda", dtype=torch.uint8)
    if case["op"] == "attn":
        s["q"] = _randn(gen, T, hq, d)
        s["o"] = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(hq, T, dtype=torch.float32, device="cuda")
    elif case["op"] == "read":
        s["k"], s["v"] = (torch.empty(T, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    else:
        fused = _randn(gen, T, hq + 2 * hkv, d)
        s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
        if case["rotate"]:
            s["q_out"] = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
            s["table_positions"] = max(lens)
            s["table"] = _table(s["table_positions"], d)
    return s


def run(s):
    """One pass; the outputs are the state's own buffers where the framework writes them."""
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"axes": _plain_axes, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[op](s)


# ------------------------------------------------------------------------------------------- the framework's calls
def _own(s, op):
    import paper_2504_20490_amd as A
    if op == "axes":
        rope = A.RopeAxes(s["table"], s["table_positions"], s["positions"], s["pair_axis"])
        A.rope_axes_qk(rope, s["q"], s["k"], s["q_out"], s["k_out"], inverse=s["case"]["inverse"])
        return {"q": s["q_out"], "k": s["k_out"]}
    cache = A.KVCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], head_dim=s["case"]["head_dim"])
    batch = A.KVBatch(s["cu_rows"], s["kv_lens"], s["page_table"], s["max_rows"])
    if op == "attn":
        if "ws" not in s:
            s["ws"] = torch.empty(A.attn_paged_workspace_bytes(cache, batch, s["q"].shape[0], s["heads"]), dtype=torch.uint8, device="cuda")
        A.attn_paged_fwd(cache, batch, s["q"], s["o"], s["lse"], s["ws"])
        return {"o": s["o"], "lse": s["lse"]}
    if op == "read":
        A.kv_cache_read(cache, batch, s["k"], s["v"])
        return {"k": s["k"], "v": s["v"]}
    if s["case"]["rotate"]:
        rope = A.RopeAxes(s["table"], s["table_positions"])
        A.kv_cache_write(cache, batch, s["k"], s["v"], rope=rope, q=s["q"], q_out=s["q_out"])
    else:
        A.kv_cache_write(cache, batch, s["k"], s["v"])
    return _written(s)


def _written(s):
    out = {name: s[name] for name in ("k_cache", "v_cache", "k_scale", "v_scale") if s[name] is not None}
    return dict(out, q=s["q_out"]) if s["case"]["rotate"] else out


# ------------------------------------------------------------------------------------------- the plain forms
def _turn(x, c, sn):
    """x [T, H, d] turned by the angles whose cosines and sines are given, [T, d / 2]; fp32, products and sums rounded one by one."""
    half = x.shape[-1] // 2
    lo, hi = x[..., :half].float(), x[..., half:].float()
    c, sn = c[:, None], sn[:, None]
    return torch.cat([lo * c - hi * sn, hi * c + lo * sn], dim=-1)


def _plain_axes(s):
    half = s["q"].shape[-1] // 2
    axis = torch.tensor(s["pair_axis"], device="cuda")
    cs = s["table"][s["positions"].long()[axis].T, torch.arange(half, device="cuda")]     # [T, half, 2]
    c, sn = cs[..., 0], -cs[..., 1] if s["case"]["inverse"] else cs[..., 1]
    return {"q": _turn(s["q"], c, sn).to(s["q"].dtype), "k": _turn(s["k"], c, sn).to(s["k"].dtype)}


def _places(s):
    """For every new row: its position in its sequence, its page and its slot there."""
    cu, lens, size = s["cu_rows"].long(), s["kv_lens"].long(), s["case"]["page_size"]
    r = torch.arange(s["k"].shape[0], device="cuda")
    seq = torch.searchsorted(cu[1:], r, right=True)
    pos = lens[seq] - cu[seq + 1] + r
    return pos, s["page_table"].long()[seq, pos // size], pos % size


def _scale_of(x):
    """The exponent of the smallest power of two from 2^-100 on that keeps |x| <= 448 over the last dimension."""
    f, e = torch.frexp(x.abs().amax(-1))
    return torch.where(f == 0, -100, (e - 9 + (f > 0.875)).clamp(min=-100))


def _plain_write(s):
    pos, page, slot = _places(s)
    k, v = s["k"].float(), s["v"].float()
    if s["case"]["rotate"]:
        cs = s["table"][pos]
        k = _turn(s["k"], cs[..., 0], cs[..., 1])
        s["q_out"].copy_(_turn(s["q"], cs[..., 0], cs[..., 1]))
    d = s["case"]["head_dim"]
    if s["case"]["cache"] == "bf16":
        s["k_cache"][page, :, slot], s["v_cache"][page, :, slot] = k.bfloat16(), v.bfloat16()
        return _written(s)
    ek, ev = _scale_of(k), _scale_of(v)
    s["k_scale"][page, :, slot], s["v_scale"][page, :, slot] = (ek + 127).to(torch.uint8), (ev + 127).to(torch.uint8)
    pad = (0, s["k_cache"].shape[-1] - d)
    bytes_of = lambda x, e: torch.nn.functional.pad(x * _pow2(-e[..., None]), pad).to(torch.float8_e4m3fn).view(torch.uint8)
    s["k_cache"].view(torch.uint8)[page, :, slot] = bytes_of(k, ek)
    s["v_cache"].view(torch.uint8)[page, :, slot] = bytes_of(v, ev)
    return _written(s)


def _pow2(e):
    """2 ** e for whole -126 <= e <= 127, exactly."""
    return (e.int() + 127 << 23).view(torch.float32)


def _values(cache, scale, index, d):
    """The fp32 values of the cache's rows at `index`."""
    x = cache[index][..., :d].float() if scale is None else cache.view(torch.uint8)[index].view(torch.float8_e4m3fn)[..., :d].float()
    return x if scale is None else x * _pow2(scale[index].int()[..., None] - 127)


def _plain_read(s):
    _, page, slot = _places(s)
    d = s["case"]["head_dim"]
    at = (page, slice(None), slot)
    return {"k": _values(s["k_cache"], s["k_scale"], at, d).bfloat16(), "v": _values(s["v_cache"], s["v_scale"], at, d).bfloat16()}


def _plain_attn(s):
    """All sequences at once, padded to the longest: scores, mask, softmax, product."""
    case = s["case"]
    hkv, d, B = case["kv_heads"], case["head_dim"], s["kv_lens"].shape[0]
    G, n, T = s["heads"] // hkv, s["max_rows"], s["q"].shape[0]
    cu, lens = s["cu_rows"].long(), s["kv_lens"].long()
    counts = cu[1:] - cu[:-1]
    r = torch.arange(n, device="cuda")
    real = r < counts[:, None]                                                   # [B, n]
    at = (cu[:-1, None] + r).clamp(max=T - 1)
    q = s["q"][at].float().view(B, n, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B * hkv, G * n, d)
    table = s["page_table"].long()
    values = lambda x: _values(s[x + "_cache"], s[x + "_scale"], table, d).permute(0, 2, 1, 3, 4).reshape(B * hkv, -1, d)
    scores = torch.bmm(q, values("k").transpose(1, 2)).mul_(1.0 / math.sqrt(d)).view(B, hkv, G, n, -1)
    pos = (lens - counts)[:, None] + r                                           # [B, n]
    seen = torch.arange(scores.shape[-1], device="cuda") <= pos[..., None]       # [B, n, L]
    scores.masked_fill_(~seen[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.bmm(scores.div_(total).view(B * hkv, G * n, -1), values("v"))
    lse = (top + total.log())[..., 0]                                            # [B, hkv, G, n]
    out = out.view(B, hkv, G, n, d).permute(0, 3, 1, 2, 4).reshape(B, n, s["heads"], d)
    return {"o": out[real].bfloat16(), "lse": lse.permute(0, 3, 1, 2).reshape(B, n, s["heads"])[real].T.contiguous()}


# ------------------------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    d, f64 = case["head_dim"], torch.float64

    def rotated(x, angle):
        z = torch.complex(x[..., :d // 2].to(f64), x[..., d // 2:].to(f64)) * torch.polar(torch.ones_like(angle), angle)[:, None]
        return torch.cat([z.real, z.imag], -1)

    theta = torch.tensor([ROPE_BASE ** (-2.0 * i / d) for i in range(d // 2)], dtype=f64, device="cuda")
    if case["op"] == "axes":
        angle = torch.stack([s["positions"][a].to(f64) * theta[i] for i, a in enumerate(s["pair_axis"])], 1)
        angle = -angle if case["inverse"] else angle
        return {"q": rotated(s["q"], angle), "k": rotated(s["k"], angle)}
    rows, lens = _geometry(case)
    size = case["page_size"]

    def cached(x, i, first, last):
        """Positions first .. last-1 of sequence i: [positions, heads, d]."""
        pages = s["page_table"][i, :-(-last // size)].long()
        flat = lambda t: t[pages].transpose(0, 1).flatten(1, 2)[:, first:last].transpose(0, 1)
        if case["cache"] == "bf16":
            return flat(s[x + "_cache"]).to(f64)
        y = flat(s[x + "_cache"].view(torch.uint8)).contiguous().view(torch.float8_e4m3fn)[..., :d].to(f64)
        return y * torch.exp2(flat(s[x + "_scale"][..., None]).to(f64) - 127.0)

    if case["op"] == "read":
        return {x: torch.cat([cached(x, i, kv - n, kv) for i, (n, kv) in enumerate(zip(rows, lens))]) for x in "kv"}
    start = 0
    if case["op"] == "attn":
        outs, lses = [], []
        group = case["heads"] // case["kv_heads"]
        for i, (n, kv) in enumerate(zip(rows, lens)):
            k, v = cached("k", i, 0, kv), cached("v", i, 0, kv)
            hidden = torch.arange(kv, device="cuda") > torch.arange(kv - n, kv, device="cuda")[:, None]
            per_head = []
            for h in range(case["heads"]):
                x = (s["q"][start:start + n, h].to(f64) @ k[:, h // group].T / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                l = torch.logsumexp(x, -1, keepdim=True)
                per_head.append((x.sub_(l).exp_() @ v[:, h // group], l[:, 0]))
            outs.append(torch.stack([o for o, _ in per_head], 1))
            lses.append(torch.stack([l for _, l in per_head]))
            start += n
        return {"o": torch.cat(outs), "lse": torch.cat(lses, 1)}
    result = {"k_cache": s["k_cache"].to(f64), "v_cache": s["v_cache"].to(f64), "q": []}
    for i, (n, kv) in enumerate(zip(rows, lens)):
        pos = torch.arange(kv - n, kv, device="cuda")
        page, slot = s["page_table"].long()[i, pos // size], pos % size
        piece = slice(start, start + n)
        turn = (lambda x: rotated(x, pos.to(f64)[:, None] * theta)) if case["rotate"] else (lambda x: x.to(f64))
        result["q"].append(turn(s["q"][piece]))
        for x, y in (("k_cache", turn(s["k"][piece])), ("v_cache", s["v"][piece].to(f64))):
            if case["cache"] == "e4m3":
                e = torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True) / 448.0)).clamp(min=-100.0)
                y = torch.nn.functional.pad(y * torch.exp2(-e), (0, _row(case) - d))
            result[x][page, :, slot] = y
        start += n
    result["q"] = torch.cat(result["q"]) if case["rotate"] else None
    result["k_scale"] = result["v_scale"] = None
    return {k: v for k, v in result.items() if k != "q" or v is not None}
