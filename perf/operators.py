"""Performance cases of the 8-bit serving operators: what a block does in 8 bits around and inside its attention.

A case is one pass through one of them, with its inputs, its weights and its cache on the GPU:

  op "norm"    rows to int8 with a scale a row, after the residual's addition and a norm (k_norm_q8)
  op "linear"  an int8 product with a scale for each token and each channel, and what follows it (k_linear_q8)
  op "cache"   new keys and values quantised into a cache as it is written, then the cache read back (k_store_q8, k_load_q8)
  op "attend"  queries over such a cache: a length for each sequence, a mask of live rows, shared key heads (k_attention_q8)

Formulas.  Rows: h = x + residual, rounded to x's type; y = (h - mean) / sqrt(mean((h - mean)^2) + eps) * weight + bias (kind "layer"),
without the mean and the bias (kind "rms"), or h itself (kind "none"); scale = max |y| / 127, q = round(y / scale).  Product: a_q w_q^T
times a_scale times w_scale, rounded to bf16; then GELU, or the residual's addition, rounded again.  Cache: 64 columns of a head and row
share a power of two 2^e <= max |x| and hold round(x 2^(6 - e)), at most 127.  Attention: softmax(q k / 8) v over the live rows
within the length, zero where there is none.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------ cases

def _norm(**kw):
    return dict(op="norm", kind="rms", rows=1374, width=1024, dtype="bf16", residual=True) | kw


def _linear(**kw):
    return dict(op="linear", rows=1041, inner=1024, outer=1024, parts=1, gelu=False, residual=False) | kw


def _cache(**kw):
    return dict(op="cache", seqs=1, held=16384, new=1374, heads=16, dtype="bf16") | kw


def _attend(**kw):
    return dict(op="attend", seqs=1, rows=1374, heads=16, kv_heads=16, held=17758, ragged=False, mask=False) | kw


def listed():
    return [
        # the camera token between two blocks: latency only
        _norm(name="norm_token", rows=1),
        # a smaller backbone run in fp32, LayerNorm with weight and bias
        _norm(name="norm_ragged_f32", kind="layer", rows=718, width=768, dtype="f32"),
        # eight frames at once
        _norm(name="norm_frames", rows=8 * 1374),
        # the first MLP product of one token
        _linear(name="linear_token", rows=1, outer=4096, gelu=True),
        # queries, keys and values of an odd frame, 12 heads
        _linear(name="linear_qkv_ragged", rows=718, inner=768, outer=2304, parts=3),
        # the second MLP product of a frame, onto the residual stream
        _linear(name="linear_frame", inner=4096, residual=True),
        # the first MLP product of eight frames
        _linear(name="linear_frames", rows=8 * 1374, outer=4096, gelu=True),
        # four streams' camera tokens into their caches, in fp32
        _cache(name="cache_tokens_f32", seqs=4, held=144, new=1, dtype="f32"),
        # a frame into a full budget, and the cache read back for what works in 16 bits
        _cache(name="cache_frame"),
        # one token each of four streams over their long caches
        _attend(name="attend_tokens", seqs=4, rows=1, held=16384, ragged=True),
        # a few tokens each of a padded batch: query heads share key heads, rows have been evicted, one sequence is empty
        _attend(name="attend_groups", seqs=8, rows=5, heads=32, kv_heads=8, held=4093, ragged=True, mask=True),
        # a frame over [cache ; frame] at the ordinary budget
        _attend(name="attend_frame"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm", "linear", "cache", "attend"])
    if op == "norm":
        width = 16 * _log_int(rng, 4, 256)
        return _norm(kind=rng.choice(["rms", "layer", "none"]), rows=_log_int(rng, 1, min(12000, 8 * 1374 * 1024 // width)), width=width,
                     dtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.7)
    if op == "linear":
        parts = rng.choice([1, 1, 3])
        inner, outer = 16 * _log_int(rng, 4, 256), parts * 8 * _log_int(rng, 8, 512 // parts)
        return _linear(rows=_log_int(rng, 1, min(12000, 8 * 1374 * 1024 * 4096 // (inner * outer))), inner=inner, outer=outer, parts=parts,
                       gelu=parts == 1 and rng.random() < 0.4, residual=parts == 1 and rng.random() < 0.5)
    seqs = _log_int(rng, 1, 8)
    if op == "cache":
        return _cache(seqs=seqs, held=_log_int(rng, 1, 16384 // seqs), new=_log_int(rng, 1, 1374), heads=rng.randint(1, 16),
                      dtype=rng.choice(["bf16", "f32"]))
    group, kv_heads = rng.choice([(1, rng.randint(1, 16)), (4, rng.randint(1, 8))])
    held = _log_int(rng, 1, 32768 // seqs)
    most = 1374 * 16 * 17758 // (seqs * group * kv_heads * held)
    return _attend(seqs=seqs, rows=_log_int(rng, 1, min(4096, most)), heads=group * kv_heads, kv_heads=kv_heads, held=held,
                   ragged=rng.random() < 0.5, mask=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows_in_8_bits(x):
    """[rows, width] fp32 -> int8 rows and a scale each."""
    scale = x.abs().amax(1) / 127
    return torch.round(x / scale[:, None]).clamp(-127, 127).to(torch.int8), scale


def _capacity(case):
    most = case["held"] + case.get("new", 0)
    return (most + 15) // 16 * 16                  # (rows of a cache: a multiple of 16)


def _fill(case, capacity, g):
    """A cache's four tensors: keys, their exponents, values, theirs."""
    heads = case.get("kv_heads", case["heads"])
    out = []
    for _ in range(2):
        x = torch.randn((case["seqs"], capacity, heads, 64), generator=g, device="cuda")
        x *= torch.exp2(torch.randint(-2, 3, (case["seqs"], capacity, heads, 1), generator=g, device="cuda") * 0.5)
        q, e = _to_blocks(x)
        out += [q.view(case["seqs"], capacity, heads * 64), e]
    return out


def prepare(case, seed):
    g = _generator(seed)
    rnd = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = dict(case)
    if case["op"] == "norm":
        t, shape = _TYPES[case["dtype"]], (case["rows"], case["width"])
        s["x"] = (rnd(*shape) * torch.exp(0.5 * rnd(case["rows"], 1))).to(t)
        s["r"] = rnd(*shape).to(t) if case["residual"] else None
        s["weight"] = None if case["kind"] == "none" else (1 + 0.1 * rnd(case["width"])).to(t)
        s["bias"] = (0.1 * rnd(case["width"])).to(t) if case["kind"] == "layer" else None
    elif case["op"] == "linear":
        s["a"], s["a_scale"] = _rows_in_8_bits(rnd(case["rows"], case["inner"]))
        s["w"], s["w_scale"] = _rows_in_8_bits(0.02 * rnd(case["outer"], case["inner"]))
        s["r"] = rnd(case["rows"], case["outer"]).bfloat16() if case["residual"] else None
        s["status"] = torch.zeros(16, dtype=torch.int32, device="cuda")
    elif case["op"] == "cache":
        t, cap = _TYPES[case["dtype"]], _capacity(case)
        s["cache"] = _fill(case, cap, g)
        shape = (case["seqs"], case["new"], case["heads"] * 64)
        s["k"], s["v"] = rnd(*shape).to(t), rnd(*shape).to(t)
        # every sequence at its own length, the first one full
        s["start"] = torch.randint(0, case["held"] + 1, (case["seqs"],), generator=g, device="cuda", dtype=torch.int32)
        s["start"][0] = case["held"]
    else:
        cap = _capacity(case)
        s["cache"] = _fill(case, cap, g)
        s["q"] = rnd(case["seqs"], case["rows"], case["heads"] * 64).bfloat16()
        s["lens"] = torch.full((case["seqs"],), case["held"], dtype=torch.int32, device="cuda")
        if case["ragged"]:
            s["lens"] = torch.randint(case["held"] // 2, case["held"] + 1, (case["seqs"],), generator=g, device="cuda", dtype=torch.int32)
            if case["seqs"] > 4:
                s["lens"][1] = 0
        s["live"] = (torch.rand((case["seqs"], cap), generator=g, device="cuda") < 0.9).to(torch.uint8) if case["mask"] else None
        s["status"] = torch.zeros(16, dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms, in 32 bits

def _pow2(n):
    """2^n in fp32 for whole n in [-126, 127]."""
    return ((n.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_blocks(x):
    """[seqs, rows, heads, 64] -> int8 of the same shape and exponents + 127 [seqs, heads, rows] uint8 (255: not finite)."""
    x = x.float()
    most = x.abs().amax(-1)
    fine = torch.isfinite(most)
    e = torch.where(fine & (most > 0), torch.frexp(torch.where(fine, most, 1.0))[1] - 1, -120).clamp(min=-120)
    q = torch.round(x * _pow2(6 - e)[..., None]).clamp(-127, 127)
    q = torch.where(fine[..., None], q, 0.0).to(torch.int8)
    return q, torch.where(fine, e + 127, 255).to(torch.uint8).transpose(1, 2).contiguous()


def _from_blocks(q, e, rows):
    """The values of the first rows: [seqs, rows, heads, 64] fp32."""
    seqs, cap, width = q.shape
    e = e[:, :, :rows].transpose(1, 2).to(torch.int32)
    step = torch.where(e == 255, float("nan"), _pow2(torch.where(e == 255, 127, e) - 133))
    return q[:, :rows].view(seqs, rows, width // 64, 64).float() * step[..., None]


def _values(q, scale):
    """What int8 rows stand for, in bf16."""
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device))


def _plain_norm(s):
    h = s["x"].float() if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype).float()
    y = h
    if s["kind"] != "none":
        y = h - h.mean(1, keepdim=True) if s["kind"] == "layer" else h
        y = y * torch.rsqrt(y.square().mean(1, keepdim=True) + EPS) * s["weight"].float()
        if s["bias"] is not None:
            y = y + s["bias"].float()
    scale = y.abs().amax(1) / 127
    q = torch.round(y / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(-127, 127)
    return _values(q.to(torch.int8), scale), scale, None if s["r"] is None else h.to(s["x"].dtype)


def _plain_linear(s):
    # (sums of products of whole numbers pass 2^24: in 64 bits)
    t = ((s["a"].double() @ s["w"].double().T).float() * s["a_scale"][:, None] * s["w_scale"]).bfloat16()
    if s["gelu"]:
        t = t.float()
        t = (0.5 * t * (1 + torch.erf(t * math.sqrt(0.5)))).bfloat16()
    if s["r"] is not None:
        return [t, (s["r"].float() + t.float()).bfloat16()]
    return list(t.view(s["rows"], s["parts"], -1).unbind(1)) if s["parts"] > 1 else [t]


def _plain_cache(s):
    rows = s["held"] + s["new"]
    kq, kx, vq, vx = s["cache"]
    shape = (s["seqs"], s["new"], s["heads"], 64)
    at = s["start"].long()[:, None] + torch.arange(s["new"], device="cuda")
    seq = torch.arange(s["seqs"], device="cuda")[:, None].expand_as(at)
    q, e = _to_blocks(s["k"].view(shape))
    kq[seq, at] = q.view(s["seqs"], s["new"], -1)
    kx.transpose(1, 2)[seq, at] = e.transpose(1, 2)
    q, e = _to_blocks(s["v"].view(shape))
    vq[seq, at] = q.view(s["seqs"], s["new"], -1)
    vx.transpose(1, 2)[seq, at] = e.transpose(1, 2)
    whole = (s["seqs"], rows, s["heads"] * 64)
    return [_from_blocks(kq, kx, rows).reshape(whole).to(s["k"].dtype), _from_blocks(vq, vx, rows).reshape(whole).to(s["k"].dtype)]


def _plain_attend(s):
    n, group = s["held"], s["heads"] // s["kv_heads"]
    kq, kx, vq, vx = s["cache"]
    live = torch.arange(n, device="cuda") < s["lens"][:, None]
    if s["live"] is not None:
        live = live & (s["live"][:, :n] != 0)
    q = s["q"].float().view(s["seqs"], s["rows"], s["kv_heads"], group, 64).permute(0, 2, 3, 1, 4).reshape(s["seqs"], s["kv_heads"], -1, 64)
    k, v = (_from_blocks(x, e, n).transpose(1, 2) for x, e in ((kq, kx), (vq, vx)))
    p = (q @ k.transpose(2, 3)) * 0.125
    p = p.masked_fill_(~live[:, None, None], float("-inf"))
    p = torch.exp(p - p.amax(-1, keepdim=True).clamp(min=-3e38))
    o = p @ v.masked_fill(~live[:, None, :, None], 0.0) / p.sum(-1, keepdim=True)
    o = torch.where(live.any(1)[:, None, None, None], o, 0.0)
    o = o.view(s["seqs"], s["kv_heads"], group, s["rows"], 64).permute(0, 3, 1, 2, 4)
    return o.reshape(s["seqs"], s["rows"], -1).bfloat16()


# ------------------------------------------------------------------ the framework's calls

def _own_norm(s):
    from paper_2603_05959_b200 import binding as B
    kind = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}[s["kind"]]
    total = None if s["r"] is None else torch.empty_like(s["x"])
    q, scale = B.k_norm_q8(s["x"], weight=s["weight"], bias=s["bias"], residual=s["r"], kind=kind, eps=EPS, sum_out=total)
    return _values(q, scale), scale, total


def _own_linear(s):
    from paper_2603_05959_b200 import binding as B
    outs = [torch.empty((s["rows"], s["outer"] // s["parts"]), dtype=torch.bfloat16, device="cuda") for _ in range(s["parts"])]
    total = None if s["r"] is None else torch.empty_like(s["r"])
    B.k_linear_q8(s["a"], s["a_scale"], s["w"], s["w_scale"], outs, gelu=s["gelu"], residual=s["r"], sum_out=total, status=s["status"])
    return outs if total is None else outs + [total]


def _own_cache(s):
    from paper_2603_05959_b200 import binding as B
    B.k_store_q8(s["cache"], s["k"], s["v"], start=s["start"])
    return list(B.k_load_q8(s["cache"], s["held"] + s["new"], dtype=s["k"].dtype))


def _own_attend(s):
    from paper_2603_05959_b200 import binding as B
    return B.k_attention_q8(s["q"], s["cache"], lens=s["lens"], live=s["live"], status=s["status"])


def run(state):
    if own:
        return {"norm": _own_norm, "linear": _own_linear, "cache": _own_cache, "attend": _own_attend}[state["op"]](state)
    return {"norm": _plain_norm, "linear": _plain_linear, "cache": _plain_cache, "attend": _plain_attend}[state["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "norm":
        n, size = case["rows"] * case["width"], {"bf16": 2, "f32": 4}[case["dtype"]]
        return {"bytes": n * size * (3 if case["residual"] else 1) + n + 4 * case["rows"], "flops": 6 * n}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inner"], case["outer"]
        return {"bytes": m * k + n * k + 4 * (m + n) + 2 * m * n * (3 if case["residual"] else 1), "flops": 2 * m * n * k}
    if case["op"] == "cache":
        width, size = case["heads"] * 64, {"bf16": 2, "f32": 4}[case["dtype"]]
        new, all_ = case["seqs"] * case["new"] * width, case["seqs"] * (case["held"] + case["new"]) * width
        return {"bytes": 2 * (new * (size + 1 + 1 / 64) + all_ * (1 + 1 / 64 + size)), "flops": 4 * new + 2 * all_}
    share = 0.75 if case["ragged"] else 1.0        # (lengths between half and all of what is held)
    if case["mask"]:
        share *= 0.9
    rows, n = case["seqs"] * case["rows"], case["held"] * share
    return {"bytes": 2 * case["seqs"] * n * case["kv_heads"] * (64 + 1) + 4 * rows * case["heads"] * 64, "flops": 4 * rows * n * case["heads"] * 64}


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_values(q, e):
    """int8 [rows, heads, 64], exponents [heads, rows] -> fp64."""
    e = e.T.double()
    return q.double() * torch.where(e == 255, float("nan"), torch.exp2(e - 133))[..., None]


def _exact_blocks(x):
    """fp64 rows [rows, heads, 64] -> what the cache holds of them, fp64."""
    most = x.abs().amax(-1, keepdim=True)
    step = torch.exp2(torch.floor(torch.log2(most.clamp(min=2.0 ** -120))) - 6)
    step = torch.where(step * 64 > most.clamp(min=2.0 ** -120), step / 2, step)      # (log2 next to a power of two)
    step = torch.where(step * 128 <= most, step * 2, step)
    return torch.clamp(torch.round(x / step), -127, 127) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        total = None
        if s["r"] is not None:
            total = h + s["r"].double()
            h = total.to(s["x"].dtype).double()
        y = h
        if case["kind"] == "layer":
            var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
            y = (h - mean) / torch.sqrt(var + EPS) * s["weight"].double() + s["bias"].double()
        elif case["kind"] == "rms":
            y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["width"] + EPS) * s["weight"].double()
        scale = y.abs().max(1).values / 127
        values = torch.round(y / scale.clamp(min=1e-300)[:, None]) * scale[:, None]
        return values, scale, total
    if case["op"] == "linear":
        t = (s["a"].double() * s["a_scale"].double()[:, None]) @ (s["w"].double() * s["w_scale"].double()[:, None]).T
        if case["gelu"]:
            t = t * torch.special.ndtr(t)
        if s["r"] is not None:
            return [t, t + s["r"].double()]
        return [p.contiguous() for p in t.chunk(case["parts"], 1)]
    if case["op"] == "cache":
        rows, heads = case["held"] + case["new"], case["heads"]
        kq, kx, vq, vx = s["cache"]
        out = []
        for q, e, new in ((kq, kx, s["k"]), (vq, vx, s["v"])):
            whole = []
            for b in range(case["seqs"]):
                x = _exact_values(q[b, :rows].view(rows, heads, 64), e[b, :, :rows])
                at = int(s["start"][b])
                x[at:at + case["new"]] = _exact_blocks(new[b].double().view(-1, heads, 64))
                whole.append(x.view(rows, heads * 64))
            out.append(torch.stack(whole))
        return out
    group, out = case["heads"] // case["kv_heads"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    kq, kx, vq, vx = s["cache"]
    for b in range(case["seqs"]):
        n = int(s["lens"][b])
        keep = torch.ones(n, dtype=torch.bool, device="cuda") if s["live"] is None else s["live"][b, :n] != 0
        if not bool(keep.any()):
            continue
        k = _exact_values(kq[b, :n].view(n, -1, 64), kx[b, :, :n])[keep]
        v = _exact_values(vq[b, :n].view(n, -1, 64), vx[b, :, :n])[keep]
        q = s["q"][b].double().view(case["rows"], case["heads"], 64)
        for h in range(case["heads"]):
            p = torch.softmax(q[:, h] @ k[:, h // group].T / 8, -1)
            out[b, :, h * 64:(h + 1) * 64] = p @ v[:, h // group]
    return out
