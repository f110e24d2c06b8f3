"""The operators of a packed K/V cache, and of per-head query/key norms, as measurable cases.

Four kinds of call:
  pack     K/V rows of a layer written to a cache held in 4 or 8 bits (`ct_pack_kv`), and the rows read
           back as the values that the cache now stands for (`ct_unpack_kv` without a rotation);
  unpack   a context put together from packed chunks: rows read back, keys rotated to their new
           positions, rows of the recompute set left out (`ct_unpack_kv`);
  attend   the newest tokens of each sequence attend over its packed cache (`ct_packed_attention`);
  norm     queries and keys of projected rows normed head by head and rotated (`ct_qk_norm_rope`).

The packed format.  Every 32 consecutive elements of a head row share a scale 2^e: the smallest e >= -117
that brings the largest magnitude to at most 1.75 * 2^emax.  An element is stored as x / 2^e rounded to
the nearest (ties to the even code) of 0, .5, 1, 1.5, 2, 3, 4, 6 (4 bits, emax = 2) or to a value with three
mantissa bits, at most 448, no step below 2^-9 (8 bits, emax = 8), and its sign.

`listed()` gives fixed cases, `draw()` more of the same ranges: one token to 131072, one sequence to 128,
one to sixteen new tokens, head sizes 64 and 128, one to sixteen query heads per KV head, both rotation styles.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

GROUP = 32
EPS = 1e-6
CUT = 1.75           # in units of 2^emax: the largest magnitude that a scale leaves
MIN_EXP = -117


# ---------------------------------------------------------------------------------- the cases
def _heads(hq, hkv, d, theta, style=0):
    return {"n_q_heads": hq, "n_kv_heads": hkv, "head_dim": d, "rope_theta": theta, "rope_style": style}


TINY = _heads(8, 2, 64, 1.0e4)
LLAMA = _heads(32, 8, 128, 5.0e5)


def _pack(name, heads, bits, n_tokens, n_rows, scattered):
    return {"name": name, "kind": "pack", **heads, "bits": bits, "n_tokens": n_tokens, "n_rows": n_rows, "scattered": scattered}


def _unpack(name, heads, bits, n_chunks, chunk_len, skip_pct, raw=False):
    return {"name": name, "kind": "unpack", **heads, "bits": bits, "n_chunks": n_chunks, "chunk_len": chunk_len,
            "skip_pct": skip_pct, "raw_keys": raw}


def _attend(name, heads, bits, n_seq, max_len, n_new, ragged):
    return {"name": name, "kind": "attend", **heads, "bits": bits, "n_seq": n_seq, "max_len": max_len, "n_new": n_new,
            "ragged": ragged}


def _norm(name, heads, n_tokens, first_pos, step):
    return {"name": name, "kind": "norm", **heads, "n_tokens": n_tokens, "first_pos": first_pos, "pos_step": step}


def listed():
    return [
        # one decoding step of 48 requests: each appends its new token to its own place in the cache
        _pack("pack_step_48", LLAMA, 4, 48, 65536, True),
        # a freshly computed chunk goes to the pool in 8 bits
        _pack("pack_chunk_2k_b8", LLAMA, 8, 2048, 4096, False),
        # the whole context of a long prompt goes to the pool in 4 bits
        _pack("pack_32k", LLAMA, 4, 32768, 32768, False),
        # eight retrieved passages make up a context; 15 % of the rows are recomputed and not read
        _unpack("unpack_8k", LLAMA, 4, 8, 1024, 15),
        # a long context of passages cached in 8 bits before their rotation, no two chunks in pool order
        _unpack("unpack_31k_b8_raw", {**LLAMA, "rope_style": 1}, 8, 23, 1387, 15, True),
        # smallest call: one short prompt on a small model; launches and latency count
        _attend("attend_1k_tiny", TINY, 4, 1, 1024, 1, False),
        # one request over the headline context
        _attend("attend_32k", LLAMA, 4, 1, 32768, 1, False),
        # a batch of requests at all stages of their answers
        _attend("attend_64x4k_ragged", LLAMA, 4, 64, 4099, 1, True),
        # drafts of four tokens checked at once, eight requests
        _attend("attend_8x16k_new4", LLAMA, 4, 8, 16384, 4, True),
        # the longest contexts, in 8 bits
        _attend("attend_2x128k_b8", LLAMA, 8, 2, 131072, 1, False),
        # a decoding step of a few requests: a handful of rows
        _norm("norm_step_7", LLAMA, 7, 20000, 311),
        # the recomputed rows of the headline context
        _norm("norm_4915", LLAMA, 4915, 3, 6),
    ]


_HEADS = [(8, 2, 64), (32, 8, 128), (16, 16, 64), (32, 4, 64), (16, 8, 128), (32, 2, 128)]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most = {k: max(w[k], most.get(k, 0)) for k in w}
    while True:
        heads = _heads(*rng.choice(_HEADS), rng.choice([1.0e4, 5.0e5]), rng.choice([0, 1]))
        bits = rng.choice([4, 4, 8])
        kind = rng.choice(["pack", "unpack", "attend", "attend", "norm"])
        if kind == "pack":
            n = _log_int(rng, 1, 32768)
            c = _pack("", heads, bits, n, (n + _log_int(rng, 1, 32768) + 31) // 32 * 32, rng.random() < 0.5)
        elif kind == "unpack":
            n = rng.randint(1, 32)
            c = _unpack("", heads, bits, n, max(1, _log_int(rng, 64, 32768) // n), rng.choice([0, 5, 15, 30, 60]),
                        rng.random() < 0.4)
        elif kind == "attend":
            c = _attend("", heads, bits, _log_int(rng, 1, 128), _log_int(rng, 1, 131072), rng.choice([1, 1, 1, 2, 3, 4, 5, 8, 16]),
                        rng.random() < 0.6)
        else:
            c = _norm("", heads, _log_int(rng, 1, 16384), rng.randint(0, 100000), rng.choice([0, 1, 7]))
        del c["name"]
        w = work(c)
        if all(w[k] <= most[k] for k in w):
            return c


# ---------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _slabs(n, row_elems):
    """Ranges of rows whose temporaries stay small."""
    step = max(1, (1 << 26) // row_elems)
    return [(lo, min(n, lo + step)) for lo in range(0, n, step)]


def _kv_rows(g, n, hkv, d):
    """K or V rows in bf16: N(0, 1) with channels of different strength, as the caches of trained models have them."""
    gain = torch.exp(0.5 * torch.randn((1, hkv, d), generator=g, device="cuda"))
    out = torch.empty((n, hkv, d), dtype=torch.bfloat16, device="cuda")
    for lo, hi in _slabs(n, hkv * d):
        out[lo:hi] = torch.randn((hi - lo, hkv, d), generator=g, device="cuda") * gain
    return out


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _sequences(case):
    """First cache row and length of each sequence; ragged ones lie one behind the other with a few rows between."""
    n, top = case["n_seq"], case["max_len"]
    if not case["ragged"]:
        step = (top + GROUP - 1) // GROUP * GROUP
        return [b * step for b in range(n)], [top] * n, n * step
    lens = [top - (b * 977) % max(1, (3 * top + 3) // 4) for b in range(n)]
    starts, at = [], 5
    for length in lens:
        starts.append(at)
        at += length + 3
    return starts, lens, (at + GROUP - 1) // GROUP * GROUP


def _inputs(case, seed):
    """Everything that goes into a pass, from the seed alone."""
    g = _generator(seed)
    rng = np.random.default_rng(seed)
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] == "norm":
        n = case["n_tokens"]
        x = torch.randn((n, (hq + 2 * hkv) * d), generator=g, device="cuda").to(torch.bfloat16)
        w = [(1 + 0.2 * torch.randn((d,), generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2)]
        return {"qkv": x, "q_weight": w[0], "k_weight": w[1], "pos": _i32(case["first_pos"] + case["pos_step"] * np.arange(n))}
    if case["kind"] == "pack":
        n = case["n_tokens"]
        k = _kv_rows(g, n, hkv, d)
        if case["scattered"]:        # a decoding step: the values are still part of the projected rows
            qkv = torch.randn((n, (hq + 2 * hkv) * d), generator=g, device="cuda").to(torch.bfloat16)
            return {"k": k, "v": qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)),
                    "rows": _i32(rng.permutation(case["n_rows"])[:n])}
        return {"k": k, "v": _kv_rows(g, n, hkv, d), "first_row": int(rng.integers(0, case["n_rows"] - n + 1))}
    if case["kind"] == "unpack":
        n_chunks, length = case["n_chunks"], case["chunk_len"]
        n = n_chunks * length
        pool = (n + GROUP - 1) // GROUP * GROUP
        order = rng.permutation(n_chunks)          # where in the pool each chunk of the context lies
        t = np.arange(n)
        rows = order[t // length] * length + t % length
        keep = np.ones(n, dtype=bool)
        keep[rng.permutation(n)[:n * case["skip_pct"] // 100]] = False
        return {"k": _kv_rows(g, pool, hkv, d), "v": _kv_rows(g, pool, hkv, d), "rows": _i32(np.where(keep, rows, -1)),
                "old_pos": None if case["raw_keys"] else _i32(t % length), "new_pos": _i32(t)}
    starts, lens, n_rows = _sequences(case)
    q = torch.randn((case["n_seq"], case["n_new"], hq, d), generator=g, device="cuda").to(torch.bfloat16)
    return {"q": q, "k": _kv_rows(g, n_rows, hkv, d), "v": _kv_rows(g, n_rows, hkv, d), "starts": starts, "lens": lens}


def prepare(case, seed):
    return _prepare_own(case, seed) if own else _prepare_plain(case, seed)


# ---------------------------------------------------------------------------------- plain forms
def _pow2(e):
    """2^e as fp32, e an integer tensor in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x, bits):
    """bf16 rows [..., d] -> codes (one byte per element) and the exponents of the groups' scales."""
    emax = 2 if bits == 4 else 8
    g = x.float().unflatten(-1, (x.shape[-1] // GROUP, GROUP))
    top = g.abs().amax(-1)
    m, p = torch.frexp(top)                      # top = m 2^p, m in [.5, 1)
    e = p - 1 - emax + (2 * m > CUT).int()
    e = torch.where(top > 0, e, MIN_EXP).clamp(min=MIN_EXP)
    y = g * _pow2(-e)[..., None]
    a = y.abs()
    if bits == 4:
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        r = (torch.round(a / step) * step).clamp(max=6)
        code = torch.zeros_like(r, dtype=torch.uint8)
        for v in (0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0):
            code += r >= v
        code += 8 * (y < 0)
    else:
        _, p = torch.frexp(a)
        step = _pow2((p - 4).clamp(min=-9))
        r = torch.round(a / step) * step
        m, p = torch.frexp(r)
        normal = ((p + 6) << 3) + (16 * m - 8).int()
        code = torch.where(r >= 2.0 ** -6, normal, (r * 512).int()).to(torch.uint8)
        code += (128 * (y < 0)).to(torch.uint8)
    return code.flatten(-2), e


def _value_table(bits):
    """What each code stands for, fp32."""
    if bits == 4:
        pos = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        pos = [(c / 8 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 1)) * 2.0 ** -6 for c in range(128)]
    return torch.tensor(pos + [-v for v in pos], dtype=torch.float32, device="cuda")


def _values(code, e, table):
    v = table[code.int()].unflatten(-1, (e.shape[-1], GROUP))
    return (v * _pow2(e)[..., None]).flatten(-2)


def _cos_sin(case, pos):
    half = case["head_dim"] // 2
    j = torch.arange(half, device="cuda", dtype=torch.float64)
    angle = pos.double()[:, None] * torch.pow(torch.tensor(case["rope_theta"], device="cuda", dtype=torch.float64), -2 * j / case["head_dim"])
    return torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]


def _rotate(x, cos, sin, style):
    half = x.shape[-1] // 2
    a, b = (x[..., :half], x[..., half:]) if style == 0 else (x[..., 0::2], x[..., 1::2])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    return torch.cat([ra, rb], -1) if style == 0 else torch.stack([ra, rb], -1).flatten(-2)


def _pack_plain_rows(x, bits):
    codes = torch.empty(x.shape, dtype=torch.uint8, device="cuda")
    exps = torch.empty((*x.shape[:-1], x.shape[-1] // GROUP), dtype=torch.int32, device="cuda")
    for lo, hi in _slabs(x.shape[0], x.shape[1] * x.shape[2]):
        codes[lo:hi], exps[lo:hi] = _quantise(x[lo:hi], bits)
    return codes, exps


def _prepare_plain(case, seed):
    s = {"case": case, "in": _inputs(case, seed)}
    i, hkv, d = s["in"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] == "norm":
        return s
    s["table"] = _value_table(case["bits"])
    if case["kind"] == "pack":
        n = case["n_rows"]
        s["cache"] = [(torch.zeros((n, hkv, d), dtype=torch.uint8, device="cuda"),
                       torch.zeros((n, hkv, d // GROUP), dtype=torch.int32, device="cuda")) for _ in range(2)]
        if "rows" in i:
            i["rows"] = i["rows"].long()
        return s
    s["cache"] = [_pack_plain_rows(i.pop(name), case["bits"]) for name in ("k", "v")]
    if case["kind"] == "unpack":
        kept = torch.nonzero(i["rows"] >= 0)[:, 0]
        s["kept"], s["from"] = kept, i["rows"][kept].long()
        s["out"] = [torch.zeros((i["rows"].shape[0], hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    return s


def _run_plain(s):
    case, i = s["case"], s["in"]
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] == "norm":
        x = i["qkv"].float().unflatten(1, (hq + 2 * hkv, d))
        cos, sin = _cos_sin(case, i["pos"])
        out = []
        for part, w in ((x[:, :hq], i["q_weight"]), (x[:, hq:hq + hkv], i["k_weight"])):
            y = part / torch.sqrt((part * part).mean(-1, keepdim=True) + EPS) * w.float()
            out.append(_rotate(y, cos, sin, case["rope_style"]).to(torch.bfloat16))
        return out[0], out[1], i["qkv"].unflatten(1, (hq + 2 * hkv, d))[:, hq + hkv:].contiguous()
    if case["kind"] == "pack":
        at = i["rows"] if "rows" in i else slice(i["first_row"], i["first_row"] + case["n_tokens"])
        out = []
        for x, (codes, exps) in zip((i["k"], i["v"]), s["cache"]):
            codes[at], exps[at] = _quantise(x, case["bits"])
            out.append(_values(codes[at], exps[at], s["table"]).to(torch.bfloat16))
        return tuple(out)
    if case["kind"] == "unpack":
        kept, src = s["kept"], s["from"]
        delta = i["new_pos"] if i["old_pos"] is None else i["new_pos"] - i["old_pos"]
        cos, sin = _cos_sin(case, delta[kept])
        k, v = (_values(codes[src], exps[src], s["table"]) for codes, exps in s["cache"])
        s["out"][0][kept] = _rotate(k, cos, sin, case["rope_style"]).to(torch.bfloat16)
        s["out"][1][kept] = v.to(torch.bfloat16)
        return tuple(s["out"])
    group, n_new = hq // hkv, case["n_new"]
    out = torch.zeros(i["q"].shape, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(i["q"].shape[:3], -math.inf, dtype=torch.float32, device="cuda")
    for b, (start, length) in enumerate(zip(i["starts"], i["lens"])):
        k, v = (_values(codes[start:start + length], exps[start:start + length], s["table"]) for codes, exps in s["cache"])
        q = i["q"][b].float().unflatten(1, (hkv, group)).permute(1, 0, 2, 3).reshape(hkv, n_new * group, d)
        x = torch.bmm(q, k.permute(1, 2, 0).contiguous()) * d ** -0.5
        x = x.unflatten(1, (n_new, group))
        if n_new > 1:                # the new token number t sees the keys up to its own place
            last = torch.arange(n_new, device="cuda") + length - n_new
            x = torch.where(torch.arange(length, device="cuda") <= last[:, None, None], x, -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.where(x > -math.inf, torch.exp(x - top), 0.0)
        total = p.sum(-1, keepdim=True)
        o = torch.bmm(p.flatten(1, 2), v.permute(1, 0, 2).contiguous()).unflatten(1, (n_new, group))
        o = torch.where(total > 0, o / total, 0.0)
        out[b] = o.permute(1, 0, 2, 3).reshape(n_new, hq, d).to(torch.bfloat16)
        lse[b] = (top + torch.log(total)).permute(1, 0, 2, 3).reshape(n_new, hq)
    return out, lse


# ---------------------------------------------------------------------------------- the framework's calls
def _prepare_own(case, seed):
    from paper_2605_24022_amd import binding as B
    i = _inputs(case, seed)
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    cfg = B.make_cfg(hq * d, hq, hkv, d, case["rope_theta"], case["rope_style"])
    s = {"case": case, "in": i, "B": B, "cfg": cfg}
    bf16 = {"dtype": torch.bfloat16, "device": "cuda"}
    if case["kind"] == "norm":
        n = case["n_tokens"]
        s["out"] = [torch.empty((n, h, d), **bf16) for h in (hq, hkv, hkv)]
        return s
    n_rows = case["n_rows"] if case["kind"] == "pack" else i["k"].shape[0]
    s["n_rows"] = n_rows
    s["cache"] = torch.empty(B.ct_packed_kv_bytes(cfg, n_rows, case["bits"]), dtype=torch.uint8, device="cuda")
    if case["kind"] == "pack":
        s["out"] = [torch.empty((case["n_tokens"], hkv, d), **bf16) for _ in range(2)]
        return s
    B.ct_pack_kv(cfg, i["k"], hkv * d, i["v"], hkv * d, n_rows, None, 0, s["cache"], n_rows, case["bits"])
    del i["k"], i["v"]
    if case["kind"] == "unpack":
        s["out"] = [torch.zeros((i["rows"].shape[0], hkv, d), **bf16) for _ in range(2)]
        return s
    s["starts"], s["lens"] = _i32(i["starts"]), _i32(i["lens"])
    s["out"] = torch.empty(i["q"].shape, **bf16)
    s["lse"] = torch.empty(i["q"].shape[:3], dtype=torch.float32, device="cuda")
    s["ws_bytes"] = B.ct_packed_attention_workspace_bytes(cfg, case["n_seq"], case["n_new"], case["max_len"])
    s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
    return s


def _run_own(s):
    case, i, B, cfg = s["case"], s["in"], s["B"], s["cfg"]
    if case["kind"] == "norm":
        B.ct_qk_norm_rope(cfg, i["qkv"], i["pos"], case["n_tokens"], i["q_weight"], i["k_weight"], EPS, *s["out"])
        return tuple(s["out"])
    if case["kind"] == "pack":
        rows, first = i.get("rows"), i.get("first_row", 0)
        B.ct_pack_kv(cfg, i["k"], i["k"].stride(0), i["v"], i["v"].stride(0), case["n_tokens"], rows, first, s["cache"],
                     s["n_rows"], case["bits"])
        B.ct_unpack_kv(cfg, s["cache"], s["n_rows"], case["bits"], rows, first, None, None, case["n_tokens"], *s["out"])
        return tuple(s["out"])
    if case["kind"] == "unpack":
        B.ct_unpack_kv(cfg, s["cache"], s["n_rows"], case["bits"], i["rows"], 0, i["old_pos"], i["new_pos"],
                       i["rows"].shape[0], *s["out"])
        return tuple(s["out"])
    B.ct_packed_attention(cfg, i["q"], case["n_seq"], case["n_new"], s["cache"], s["n_rows"], case["bits"], s["starts"],
                          s["lens"], case["max_len"], s["out"], s["lse"], s["ws"], s["ws_bytes"])
    return s["out"], s["lse"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------- the definition in 64 bits
def _stored64(x, bits):
    """What bf16 rows are held as: nearest member of the code's value list, the lower neighbour's or the upper
    one's, whichever has the even place in the list where both are as near."""
    if bits == 4:
        values, limit = [0, 0.5, 1, 1.5, 2, 3, 4, 6], 7.0
    else:
        values = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1]
        limit = 448.0
    values = torch.tensor(values, dtype=torch.float64, device="cuda")
    g = x.double().unflatten(-1, (-1, GROUP))
    # (by a tensor: division by a number is a product with its reciprocal on the device, and off by a bit at the border)
    m, p = torch.frexp(g.abs().amax(-1) / torch.tensor([limit], dtype=torch.float64, device="cuda"))
    e = torch.where(m == 0.5, p - 1, p)                     # the smallest with max <= limit 2^e
    e = torch.where(m == 0, MIN_EXP, e).clamp(min=MIN_EXP)
    scale = ((e.long() + 1023) << 52).view(torch.float64)[..., None]        # 2^e, to the last bit
    a = g.abs() / scale
    hi = torch.searchsorted(values, a).clamp(max=len(values) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = (values[hi] - a).abs(), (a - values[lo]).abs()
    pick = torch.where(up < down, hi, torch.where(down < up, lo, torch.where(hi % 2 == 0, hi, lo)))
    return (torch.sign(g) * values[pick] * scale).flatten(-2)


def _turn64(x, pos, theta, style):
    """Pairs as complex numbers times e^(i pos omega)."""
    d = x.shape[-1]
    omega = theta ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
    turn = torch.polar(torch.ones((), device="cuda", dtype=torch.float64), pos.double()[:, None] * omega)[:, None, :]
    pairs = x.unflatten(-1, (2, d // 2)).transpose(-1, -2) if style == 0 else x.unflatten(-1, (d // 2, 2))
    y = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
    return y.transpose(-1, -2).flatten(-2) if style == 0 else y.flatten(-2)


def exact(case, seed):
    i = _inputs(case, seed)
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    theta, style = case["rope_theta"], case["rope_style"]
    if case["kind"] == "norm":
        x = i["qkv"].double().unflatten(1, (-1, d))
        unit = x * torch.rsqrt(x.pow(2).sum(-1, keepdim=True) / d + EPS)
        return (_turn64(unit[:, :hq] * i["q_weight"].double(), i["pos"], theta, style),
                _turn64(unit[:, hq:hq + hkv] * i["k_weight"].double(), i["pos"], theta, style), x[:, hq + hkv:])
    if case["kind"] == "pack":
        return tuple(torch.cat([_stored64(x[lo:hi], case["bits"]) for lo, hi in _slabs(x.shape[0], hkv * d)])
                     for x in (i["k"], i["v"]))
    if case["kind"] == "unpack":
        out = [torch.zeros((i["rows"].shape[0], hkv, d), dtype=torch.float64, device="cuda") for _ in range(2)]
        kept = i["rows"] >= 0
        src = i["rows"][kept].long()
        turn = i["new_pos"] - (0 if i["old_pos"] is None else i["old_pos"])
        out[0][kept] = _turn64(_stored64(i["k"][src], case["bits"]), turn[kept], theta, style)
        out[1][kept] = _stored64(i["v"][src], case["bits"])
        return tuple(out)
    n_new = case["n_new"]
    out = torch.zeros(i["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(i["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b, (start, length) in enumerate(zip(i["starts"], i["lens"])):
        k, v = (_stored64(i[name][start:start + length], case["bits"]).transpose(0, 1).contiguous() for name in ("k", "v"))
        q = i["q"][b].double().unflatten(1, (hkv, -1)).transpose(0, 1).flatten(1, 2)        # [hkv, n_new * group, d]
        x = torch.bmm(k, q.transpose(1, 2).contiguous()).unflatten(2, (n_new, -1)) / math.sqrt(d)
        for t in range(n_new):
            n = length - n_new + t + 1          # keys that this token sees
            if n > 0:
                lse[b, t] = torch.logsumexp(x[:, :n, t], 1).flatten()
                p = torch.softmax(x[:, :n, t], 1).transpose(1, 2).contiguous()
                out[b, t] = torch.bmm(p, v[:, :n].contiguous()).flatten(0, 1)
    return out, lse


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    hq, hkv, d = case["n_q_heads"], case["n_kv_heads"], case["head_dim"]
    if case["kind"] == "norm":
        elems = case["n_tokens"] * (hq + 2 * hkv) * d
        return {"bytes": 4 * elems + 4 * d + 4 * case["n_tokens"], "flops": 7.0 * case["n_tokens"] * (hq + hkv) * d}
    row = 2 * hkv * d                                          # elements of K and V per token
    packed = row * case["bits"] // 8 + row // GROUP           # bytes of them in the cache
    if case["kind"] == "pack":
        n = case["n_tokens"]
        return {"bytes": n * (4 * row + 2 * packed + (8 if case["scattered"] else 0)), "flops": 4.0 * n * row}
    if case["kind"] == "unpack":
        n = case["n_chunks"] * case["chunk_len"]
        kept = n - n * case["skip_pct"] // 100
        return {"bytes": kept * (packed + 2 * row) + n * (8 if case["raw_keys"] else 12), "flops": 4.0 * kept * row}
    _, lens, _ = _sequences(case)
    keys, n_seq, n_new = sum(lens), case["n_seq"], case["n_new"]
    seen = sum(max(0, length - n_new + t + 1) for length in lens for t in range(n_new))
    return {"bytes": keys * packed + n_seq * n_new * hq * (4 * d + 4) + 8 * n_seq, "flops": 4.0 * hq * d * seen}
