"""Packed caches on the GPU: rows written and read back bit for bit, keys rotated on the way, attention of the newest
tokens over them, per-head norms, and these calls together as a request uses them, against the oracle in 64 bits.

Bounds.  A rounding to bf16 is off by at most 2^-8 of the value (half a step).  Rotations: hardware sine and cosine of an
fp32 angle in turns are good to 2^-19.5 together, so a rotated pair (a, b) gets 2^-18 (|a| + |b|) besides.  Attention:
each probability enters the product in bf16, which moves an output by at most 2^-8 sum p |v|; a score of D exact
products added in fp32 is off by at most D 2^-24 sum |q k| scale, and the exponential and the sums by less than 2^-18."""
import numpy as np
import pytest
import torch

from oracle import ct_oracle as O
from paper_2605_24022_amd import binding as B
from paper_2605_24022_amd import workloads as W
from tests.gpu_util import assert_close, bits_of, dev_bf16, dev_i32, f64_of, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available()
    B.load()
    torch.cuda.set_device(0)


def _cfg(hq, hkv, d, theta=1e4, style=0, scale=0.0):
    return B.make_cfg(hq * d, hq, hkv, d, theta, style, scale)


def _bits(rng, *shape, spread=1.0):
    """bf16 patterns of normal numbers whose groups differ in magnitude."""
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal((*shape[:-1], 1)))
    return W.f32_to_bf16_bits(x.astype(np.float32))


def _cache(cfg, n_rows, bits, fill=0xff):
    """A cache whose bytes are all NaN until rows are written."""
    return torch.full((B.ct_packed_kv_bytes(cfg, n_rows, bits),), fill, dtype=torch.uint8, device="cuda")


def _pack(cfg, k, v, cache, n_rows, bits, rows=None, first=0):
    kd, vd = dev_bf16(k), dev_bf16(v)
    B.ct_pack_kv(cfg, kd, kd.stride(0), vd, vd.stride(0), k.shape[0], rows, first, cache, n_rows, bits)


def _read(cfg, cache, n_rows, bits, hkv, d):
    k, v = (torch.empty((n_rows, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ct_unpack_kv(cfg, cache, n_rows, bits, None, 0, None, None, n_rows, k, v)
    return f64_of(k), f64_of(v)


def _same(got, want, what):
    """Equal values, NaN where NaN is expected."""
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    bad = ~((got == want) | np.isnan(want))
    assert not bad.any(), f"{what}: {bad.sum()} values differ, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


def _attend(cfg, q, n_seq, n_new, cache, n_rows, bits, starts, lens, max_len, out):
    need = B.ct_packed_attention_workspace_bytes(cfg, n_seq, n_new, max_len)
    ws = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device="cuda")
    B.ct_packed_attention(cfg, q, n_seq, n_new, cache, n_rows, bits, dev_i32(starts), dev_i32(lens), max_len, out, None, ws, need)


SHAPES = [(2, 64, 4), (2, 64, 8), (8, 128, 4), (8, 128, 8), (1, 128, 4), (3, 64, 4), (5, 128, 8)]


# ---------------------------------------------------------------------------------- write and read back
@pytest.mark.parametrize("hkv,d,bits", SHAPES)
@pytest.mark.parametrize("n", [1, 31, 33, 100])
def test_rows_come_back_as_the_values_they_stand_for(hkv, d, bits, n):
    say(f"pack hkv={hkv} d={d} bits={bits} n={n}")
    rng = np.random.default_rng([n, hkv, d, bits])
    cfg, n_rows = _cfg(hkv, hkv, d), 192
    cache = _cache(cfg, n_rows, bits)
    k0, v0 = _bits(rng, n_rows, hkv, d), _bits(rng, n_rows, hkv, d)
    _pack(cfg, k0, v0, cache, n_rows, bits)
    wk, wv = (O.packed_values(W.bf16_bits_to_f64(x), bits) for x in (k0, v0))
    gk, gv = _read(cfg, cache, n_rows, bits, hkv, d)
    _same(gk, wk, "K, whole cache")
    _same(gv, wv, "V, whole cache")
    # rows anywhere, some of them nowhere; a run from an odd row on
    rows = rng.permutation(n_rows)[:n].astype(np.int32)
    if n > 4:
        rows[[0, 2, 3]] = [-1, n_rows, -2 ** 31]
    for first in (None, 37):
        k1, v1 = _bits(rng, n, hkv, d, spread=3.0), _bits(rng, n, hkv, d, spread=3.0)
        at = rows if first is None else first + np.arange(n)
        _pack(cfg, k1, v1, cache, n_rows, bits, dev_i32(rows) if first is None else None, first or 0)
        ok = (at >= 0) & (at < n_rows)
        wk[at[ok]], wv[at[ok]] = (O.packed_values(W.bf16_bits_to_f64(x[ok]), bits) for x in (k1, v1))
        gk, gv = _read(cfg, cache, n_rows, bits, hkv, d)
        _same(gk, wk, f"K, rows {first}")
        _same(gv, wv, f"V, rows {first}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
def test_every_bf16_number_beside_every_scale_border(d, bits):
    """All finite bf16 numbers as elements of groups whose largest magnitude lies on, below and above the border of a
    scale, the smallest and the largest scales, zeros of both signs, infinities and NaN."""
    say(f"pack values d={d} bits={bits}")
    every = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    every = every[(every & 0x7f80) != 0x7f80]
    every = np.concatenate([every, every[: -every.size % 31]]).reshape(-1, 31)
    exps = np.array([0, 8, 9, 10, 100, 127, 128, 140, 252, 253, 254])
    tops = ((exps[:, None] << 7) | np.array([0, 0x5f, 0x60, 0x61, 0x7f])[None]).ravel().astype(np.uint16)
    groups = [np.concatenate([[t], np.where((e & 0x7fff) <= t, e, t)]) for t in tops for e in every[:: 37]]
    groups += [np.concatenate([[0x8000], e & 0x8000]) for e in every[:4]]
    groups += [np.concatenate([[bad], e]) for bad in (0x7f80, 0xff80, 0x7fc0, 0xffff, 0x7f81) for e in every[300:303]]
    x = np.array(groups, dtype=np.uint16)
    per_row = d // 32
    n = x.shape[0] // per_row // 32 * 32
    x = x[: n * per_row].reshape(n, 1, d)
    tail = np.array(groups[-15:] + groups[-15 - 4: -15], dtype=np.uint16)      # (cut off above: the special ones)
    x[: tail.shape[0] // per_row] = tail[: tail.shape[0] // per_row * per_row].reshape(-1, 1, d)
    cfg = _cfg(1, 1, d)
    cache = _cache(cfg, n, bits)
    _pack(cfg, x, x[::-1].copy(), cache, n, bits)
    gk, gv = _read(cfg, cache, n, bits, 1, d)
    want = O.packed_values(W.bf16_bits_to_f64(x), bits)
    assert np.isnan(want).any()
    _same(gk, want, "K")
    _same(gv, want[::-1], "V")


@pytest.mark.parametrize("d,bits", [(64, 8), (128, 4)])
def test_rows_inside_projected_rows(d, bits):
    """Strides: keys and values taken out of projected [q|k|v] rows."""
    hq, hkv, n, n_rows = 4, 2, 45, 64
    say(f"pack strided d={d} bits={bits}")
    rng = np.random.default_rng(d)
    qkv = _bits(rng, n, (hq + 2 * hkv) * d)
    x = dev_bf16(qkv)
    cfg = _cfg(hq, hkv, d)
    cache = _cache(cfg, n_rows, bits)
    B.ct_pack_kv(cfg, x[:, hq * d:], x.stride(0), x[:, (hq + hkv) * d:], x.stride(0), n, None, 3, cache, n_rows, bits)
    gk, gv = _read(cfg, cache, n_rows, bits, hkv, d)
    want = W.bf16_bits_to_f64(qkv).reshape(n, -1, d)
    _same(gk[3:3 + n], O.packed_values(want[:, hq:hq + hkv], bits), "K")
    _same(gv[3:3 + n], O.packed_values(want[:, hq + hkv:], bits), "V")
    assert np.isnan(gk[:3]).all() and np.isnan(gv[3 + n:]).all()               # not written


@pytest.mark.parametrize("hkv,d,bits", [(2, 64, 4), (8, 128, 8)])
def test_blocks_of_rows_are_copied_as_bytes(hkv, d, bits):
    """Rows 64 to 127 of one cache become rows 32 to 95 of another, by way of pinned host memory."""
    say(f"packed blocks copied hkv={hkv} d={d} bits={bits}")
    rng = np.random.default_rng([hkv, d, bits])
    cfg, per = _cfg(hkv, hkv, d), B.ct_packed_kv_bytes(_cfg(hkv, hkv, d), 32, bits)
    one, other = _cache(cfg, 160, bits), _cache(cfg, 128, bits)
    k, v = _bits(rng, 160, hkv, d), _bits(rng, 160, hkv, d)
    _pack(cfg, k, v, one, 160, bits)
    assert B.ct_packed_kv_bytes(cfg, 64, bits) == 2 * per
    host = torch.empty(2 * per, dtype=torch.uint8, pin_memory=True)
    host.copy_(one[2 * per:4 * per])
    other[per:3 * per].copy_(host)
    gk, gv = _read(cfg, other, 128, bits, hkv, d)
    for got, x in ((gk, k), (gv, v)):
        _same(got[32:96], O.packed_values(W.bf16_bits_to_f64(x[64:128]), bits), "copied rows")
        assert np.isnan(got[:32]).all() and np.isnan(got[96:]).all()


def _rope_bound(want, d, style):
    a = np.abs(want)
    if style == 0:
        pair = np.concatenate([a[..., : d // 2] + a[..., d // 2:]] * 2, axis=-1)
    else:
        pair = np.repeat(a[..., 0::2] + a[..., 1::2], 2, axis=-1)
    return 2.0 ** -8 * a + 2.0 ** -18 * 1.5 * pair      # (|a| + |b| of the rotated pair is at least 0.7 of the unrotated one's)


@pytest.mark.parametrize("hkv,d,bits", SHAPES)
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("raw", [False, True])
def test_rows_read_back_and_rotated(hkv, d, bits, style, raw):
    say(f"unpack hkv={hkv} d={d} bits={bits} style={style} raw={raw}")
    rng = np.random.default_rng([hkv, d, bits, style])
    n_rows, n = 160, 217
    cfg = _cfg(hkv, hkv, d, 5e5, style)
    cache = _cache(cfg, n_rows, bits)
    k, v = _bits(rng, n_rows, hkv, d), _bits(rng, n_rows, hkv, d)
    _pack(cfg, k, v, cache, n_rows, bits)
    rows = rng.integers(0, n_rows, n).astype(np.int32)                         # some more than once
    rows[rng.permutation(n)[:40]] = -1
    rows[:2] = [n_rows, -7]
    old = rng.integers(0, 4096, n).astype(np.int32)
    new = rng.integers(0, 131072, n).astype(np.int32)
    new[5:9] = old[5:9]
    mark = torch.full((n, hkv, d), 123.0, dtype=torch.bfloat16, device="cuda")
    kd, vd = mark.clone(), mark.clone()
    B.ct_unpack_kv(cfg, cache, n_rows, bits, dev_i32(rows), 0, None if raw else dev_i32(old), dev_i32(new), n, kd, vd)
    gk, gv = f64_of(kd), f64_of(vd)
    ok = (rows >= 0) & (rows < n_rows)
    assert (gk[~ok] == 123).all() and (gv[~ok] == 123).all()
    _same(gv[ok], O.packed_values(W.bf16_bits_to_f64(v), bits)[rows[ok]], "V")
    kept = O.packed_values(W.bf16_bits_to_f64(k), bits)[rows[ok]]
    want = O.rotate(kept, (new if raw else new - old)[ok], 5e5, style)
    assert (np.abs(gk[ok] - want) <= _rope_bound(want, d, style)).all()
    if not raw:
        still = [i for i in range(5, 9) if ok[i]]
        _same(gk[still], O.packed_values(W.bf16_bits_to_f64(k), bits)[rows[still]], "K that stays where it was")


# ---------------------------------------------------------------------------------- attention
def _held_to_oracle(got, q, k, v, what, scale=None):
    """One sequence's outputs [n_new, Hq, D] against the oracle.  (An absolute bound of unit-scale data does not fit here: at
    magnitude 8 the rounding of the result alone is up to 8 * 2^-8 = 0.031.)"""
    d = q.shape[-1]
    scale = 1 / np.sqrt(d) if scale is None else scale
    want, lse, weight = O.packed_attention(q, k, v, scale)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    reach = np.nan_to_num(np.abs(k)).max() * np.abs(q).sum(-1).max() * scale * d * 2.0 ** -24 if k.size else 0.0
    bound = 2.0 ** -8 * (np.abs(want) + weight) + (2.0 ** -18 + 2 * reach) * weight
    excess = np.abs(np.where(nan, 0, got) - np.where(nan, 0, want)) - np.where(nan, 0, bound)
    assert excess.max() <= 0, f"{what}: beyond its bound by {excess.max()}"
    return want, lse, reach


def _check_attention(hq, hkv, d, bits, n_new, lens, starts, n_rows, seed=1, max_len=None, scale=0.0, spread=0.5, edit=None,
                     with_lse=True):
    say(f"packed attention heads={hq}/{hkv} d={d} bits={bits} n_new={n_new} lens={lens[:8]} starts={starts[:8]} rows={n_rows}")
    rng = np.random.default_rng([seed, hq, d, bits, n_new, len(lens)])
    cfg = _cfg(hq, hkv, d, scale=scale)
    cache = _cache(cfg, n_rows, bits)
    k, v = _bits(rng, n_rows, hkv, d, spread=spread), _bits(rng, n_rows, hkv, d, spread=spread)
    if edit is not None:
        edit(k, v)
    inside = np.zeros(n_rows, dtype=bool)
    for s, n in zip(starts, lens):
        inside[s:s + n] = True
    rows = np.flatnonzero(inside).astype(np.int32)      # nothing else is written: the rest of the cache reads as NaN
    if rows.size:
        _pack(cfg, k[rows], v[rows], cache, n_rows, bits, dev_i32(rows))
    n_seq = len(lens)
    q = _bits(rng, n_seq, n_new, hq, d, spread=0.3)
    max_len = max(lens) if max_len is None else max_len
    need = B.ct_packed_attention_workspace_bytes(cfg, n_seq, n_new, max_len)
    ws = torch.full((max(need, 256) + 256,), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((n_seq, n_new, hq, d), 77.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_seq, n_new, hq), 77.0, dtype=torch.float32, device="cuda")
    args = (cfg, dev_bf16(q), n_seq, n_new, cache, n_rows, bits, dev_i32(starts), dev_i32(lens), max_len)
    B.ct_packed_attention(*args, out, lse if with_lse else None, ws, need)
    assert (ws[max(need, 256):] == 0xff).all(), "wrote behind its workspace"
    got, got_lse = f64_of(out), lse.cpu().numpy().astype(np.float64)
    if not with_lse:
        assert (got_lse == 77).all()
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(x), bits) for x in (k, v))
    qv = W.bf16_bits_to_f64(q)
    real_scale = scale or 1 / np.sqrt(d)
    for b, (s, n) in enumerate(zip(starts, lens)):
        want, want_lse, reach = _held_to_oracle(got[b], qv[b], kv[s:s + n], vv[s:s + n], f"sequence {b}", real_scale)
        nan = np.isnan(want)
        if with_lse:
            fin = np.isfinite(want_lse)
            assert np.array_equal(got_lse[b][~fin & ~np.isnan(want_lse)], want_lse[~fin & ~np.isnan(want_lse)])
            assert np.array_equal(np.isnan(got_lse[b]), np.isnan(want_lse))
            assert (np.abs(got_lse[b][fin] - want_lse[fin]) <= reach + 2.0 ** -20 * (8 + np.abs(want_lse[fin]))).all()
        if n and not nan.any():
            seen = np.abs(want).sum(-1) > 0
            rel = np.sqrt(((got[b] - want) ** 2).sum(-1) / np.maximum((want ** 2).sum(-1), 1e-30))[seen]
            assert rel.size == 0 or rel.max() <= 1e-2, f"sequence {b}: row off by {rel.max()} of its norm"
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    B.ct_packed_attention(*args, out2, lse2 if with_lse else None, ws, need)
    assert np.array_equal(bits_of(out), bits_of(out2)), "a second call gives other bits"
    return need


HEADS = [(8, 2, 64), (16, 16, 64), (32, 8, 128), (16, 8, 128), (8, 1, 128), (16, 1, 64), (16, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("bits", [4, 8])
def test_single_tokens_at_all_lengths(hq, hkv, d, bits):
    """One new token per sequence: empty ones, one row, both sides of the 32-row block and of a part, any start."""
    lens = [0, 1, 2, 31, 32, 33, 64, 95, 255, 257, 300, 0]
    starts, at = [], 3
    for i, n in enumerate(lens):
        starts.append(at)
        at += n + (i % 3)
    _check_attention(hq, hkv, d, bits, 1, lens, starts, (at + 31) // 32 * 32)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("n_new", [2, 5, 16])
@pytest.mark.parametrize("bits", [4, 8])
def test_several_new_tokens(hq, hkv, d, n_new, bits):
    """Causal among the new ones, blocks that the earlier do not see, more new tokens than rows; up to 256 columns."""
    lens = [1, 3, 16, 32, 40, 129, 333]
    starts = [0, 1, 7, 32, 64, 150, 290]
    _check_attention(hq, hkv, d, bits, n_new, lens, starts, 640)


def test_most_new_tokens():
    _check_attention(8, 4, 64, 4, 64, [63, 64, 65, 500], [0, 70, 140, 211], 736)


@pytest.mark.parametrize("hq,hkv,d,bits,n_new,lens", [
    (8, 2, 64, 4, 1, [5000]), (32, 8, 128, 4, 1, [8191]), (32, 8, 128, 8, 3, [4097, 0, 200]), (16, 1, 128, 4, 1, [20000]),
    (16, 8, 128, 8, 1, [3001, 7, 2999, 1000]), (8, 2, 64, 8, 6, [6000, 1, 257])])
def test_key_ranges_in_parts(hq, hkv, d, bits, n_new, lens):
    """Long sequences, whose key range several workgroups divide, beside short ones that one of them finishes."""
    starts = (13 + np.cumsum([0] + lens[:-1])).tolist()
    need = _check_attention(hq, hkv, d, bits, n_new, lens, starts, (sum(lens) + 13 + 31) // 32 * 32)
    assert need > 0


def test_bound_above_the_lengths():
    """The key range is divided for max_len; the lengths themselves are on the device."""
    _check_attention(32, 8, 128, 4, 2, [100, 900, 0], [40, 200, 0], 32768, max_len=30000)


@pytest.mark.parametrize("n_seq", [3, 5, 7, 9, 11, 13, 17, 20, 24, 31, 33, 47, 49])
@pytest.mark.parametrize("bits,n_new", [(4, 1), (8, 20)])
def test_batches_divided_one_two_and_three_to_a_unit(n_seq, bits, n_new):
    lens = [1500 - 211 * i % 1400 for i in range(n_seq)]
    starts = np.concatenate([[0], np.cumsum(lens)[:-1]]).tolist()
    _check_attention(8, 8, 64, bits, n_new, lens, starts, (sum(lens) + 31) // 32 * 32)


def test_many_sequences():
    lens = [(37 * i) % 150 for i in range(300)]
    starts = np.concatenate([[0], np.cumsum(lens)[:-1]]).tolist()
    _check_attention(8, 2, 64, 4, 1, lens, starts, (sum(lens) + 31) // 32 * 32)


@pytest.mark.parametrize("n_seq", [17, 32, 33, 64, 65, 200, 256, 257])
def test_batches_in_the_order_of_their_lengths(n_seq):
    """Long batches take their sequences in another order than they come, 16 of them do not: every sequence gets the same bits."""
    hq, hkv, d, n_rows, max_len = 16, 16, 64, 4096, 2100
    say(f"order of lengths n_seq={n_seq}")
    rng = np.random.default_rng(n_seq)
    cfg = _cfg(hq, hkv, d)
    cache = _cache(cfg, n_rows, 4)
    _pack(cfg, _bits(rng, n_rows, hkv, d, spread=0.3), _bits(rng, n_rows, hkv, d, spread=0.3), cache, n_rows, 4)
    q = dev_bf16(_bits(rng, n_seq, 1, hq, d, spread=0.3))
    # many of equal length, empty ones, some at and beyond the bound, one below zero, one whose start is no row
    lens = rng.choice([0, 1, 31, 32, 33, 70, 500, 1999, 2100], n_seq)
    lens[[2, 5, 11]] = 5000, -7, 64
    starts = rng.integers(0, n_rows - max_len, n_seq)
    starts[11] = n_rows
    got = torch.full_like(q, float("nan"))
    _attend(cfg, q, n_seq, 1, cache, n_rows, 4, starts, lens, max_len, got)
    want = torch.full_like(q, float("nan"))
    for b in range(0, n_seq, 16):
        b = min(b, n_seq - 16)
        e = b + 16
        _attend(cfg, q[b:e], e - b, 1, cache, n_rows, 4, starts[b:e], lens[b:e], max_len, want[b:e])
    torch.cuda.synchronize()
    assert not torch.isnan(got).any()
    got, want = bits_of(got), bits_of(want)
    bad = [b for b in range(n_seq) if not np.array_equal(got[b], want[b])]
    assert not bad, f"sequences {bad[:8]} of lengths {lens[bad[:8]]} differ"


def test_sequences_may_share_rows():
    """Two requests over one prompt: overlapping ranges of the cache."""
    _check_attention(16, 8, 128, 4, 1, [500, 500, 200], [10, 10, 300], 512)


@pytest.mark.parametrize("scale,spread", [(2.0, 0.5), (0.01, 0.5), (0.0, 2.5)])
def test_peaked_and_flat_rows(scale, spread):
    """One key takes all the weight, all keys share it, keys and values of very different size."""
    _check_attention(32, 8, 128, 8, 2, [700, 33], [5, 720], 768, scale=scale, spread=spread)


@pytest.mark.parametrize("hq,hkv,d,bits", [(8, 2, 64, 4), (8, 2, 64, 8), (32, 8, 128, 4), (16, 8, 128, 8)])
@pytest.mark.parametrize("bad", [0x7f80, 0xff80, 0x7fc0])
def test_infinities_and_nan_reach_those_who_see_them(hq, hkv, d, bits, bad):
    """An infinity or a NaN in the newest tokens' keys or values: NaN for the tokens that see it (for a value, in its 32
    dimensions), nothing for the earlier ones; outside the sequence, nothing at all."""
    def edit(k, v):
        v[16 + 299, 0, 33] = bad          # the last but one token of sequence 0
        v[16 + 300, 1, 5] = bad           # its last
        k[400 + 69, 0, 1] = bad           # the last but one of sequence 1
        v[600 + 3, 1, 40] = bad           # an early row of sequence 2: everybody sees it
        v[15], k[15], v[397], k[396] = bad, bad, bad, bad
    _check_attention(hq, hkv, d, bits, 4, [301, 71, 50, 3], [16, 400, 600, 394], 704, edit=edit)


@pytest.mark.parametrize("n_new,lens,nan_keys", [
    (1, [1, 40], [0]),                                # nothing but a NaN
    (1, [128, 40], list(range(32, 64))),              # all that one wave sees
    (2, [2, 3], [1]),                                 # the earlier token sees none of it
    (1, [6000, 40], list(range(2048, 4096))),         # all that one part of the key range holds
    (1, [6000, 40], list(range(6000)))])
def test_keys_that_are_all_nan(n_new, lens, nan_keys):
    """Scores that are all NaN leave no maximum behind: output and log-sum-exp are NaN all the same."""
    def edit(k, v):
        k[5 + np.array(nan_keys)] = 0x7fc0
    _check_attention(8, 2, 64, 4, n_new, lens, [5, 6050], 6112, edit=edit)


def test_without_lse():
    _check_attention(8, 2, 64, 4, 1, [3000, 20], [0, 3000], 3040, with_lse=False)


def test_lengths_and_starts_that_do_not_fit_are_cut():
    """Lengths above max_len or past the cache's end are cut, negative starts and lengths are empty sequences."""
    hq, hkv, d, bits, n_rows = 8, 2, 64, 4, 256
    say("packed attention, cut lengths")
    rng = np.random.default_rng(3)
    cfg = _cfg(hq, hkv, d)
    cache = _cache(cfg, n_rows, bits)
    k, v = _bits(rng, n_rows, hkv, d), _bits(rng, n_rows, hkv, d)
    _pack(cfg, k, v, cache, n_rows, bits)
    starts, lens = [0, 200, -5, 3, 300, 2 ** 31 - 1], [1000, 100, 10, -4, 10, 2 ** 31 - 1]
    q = _bits(rng, 6, 1, hq, d)
    out = torch.empty((6, 1, hq, d), dtype=torch.bfloat16, device="cuda")
    _attend(cfg, dev_bf16(q), 6, 1, cache, n_rows, bits, starts, lens, 128, out)
    got = f64_of(out)
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(x), bits) for x in (k, v))
    for b, (s, n) in enumerate([(0, 128), (200, 56)]):
        _held_to_oracle(got[b], W.bf16_bits_to_f64(q)[b], kv[s:s + n], vv[s:s + n], f"sequence {b}")
    assert (got[2:] == 0).all()


def test_offsets_beyond_four_gigabytes():
    """Rows far behind the first 4 GiB of the cache."""
    hq, hkv, d, bits = 32, 8, 128, 8
    cfg, n_rows, n = _cfg(hq, hkv, d), 2100000 // 32 * 32, 70
    first = n_rows - n - 1
    say(f"packed cache of {B.ct_packed_kv_bytes(cfg, n_rows, bits)} bytes")
    assert (first // 32) * (B.ct_packed_kv_bytes(cfg, 32, bits)) > 1 << 32
    cache = torch.empty(B.ct_packed_kv_bytes(cfg, n_rows, bits), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(9)
    k, v, q = _bits(rng, n, hkv, d), _bits(rng, n, hkv, d), _bits(rng, 1, 1, hq, d)
    _pack(cfg, k, v, cache, n_rows, bits, None, first)
    kd, vd = (torch.empty((n, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ct_unpack_kv(cfg, cache, n_rows, bits, None, first, None, None, n, kd, vd)
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(x), bits) for x in (k, v))
    _same(f64_of(kd), kv, "K")
    _same(f64_of(vd), vv, "V")
    out = torch.empty((1, 1, hq, d), dtype=torch.bfloat16, device="cuda")
    _attend(cfg, dev_bf16(q), 1, 1, cache, n_rows, bits, [first], [n], n, out)
    _held_to_oracle(f64_of(out)[0], W.bf16_bits_to_f64(q)[0], kv, vv, "attention")


# ---------------------------------------------------------------------------------- norms of queries and keys
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (16, 16, 64), (32, 8, 128), (16, 1, 128), (2, 1, 64)])
@pytest.mark.parametrize("n", [1, 3, 130])
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_norm_and_rotation(hq, hkv, d, n, style, eps):
    say(f"qk norm heads={hq}/{hkv} d={d} n={n} style={style} eps={eps}")
    rng = np.random.default_rng([hq, d, n, style])
    x = _bits(rng, n, (hq + 2 * hkv), d, spread=2.0).reshape(n, -1)
    qw, kw = (W.f32_to_bf16_bits((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)) for _ in range(2))
    pos = rng.integers(0, 1 << 20, n).astype(np.int32)
    cfg = _cfg(hq, hkv, d, 5e5, style)
    q, k, v = (torch.full((n + 1, h, d), 55.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    args = (cfg, dev_bf16(x), dev_i32(pos), n, dev_bf16(qw), dev_bf16(kw), eps)
    B.ct_qk_norm_rope(*args, q, k, v)
    want = O.qk_norm_rope(W.bf16_bits_to_f64(x), pos, W.bf16_bits_to_f64(qw), W.bf16_bits_to_f64(kw), np.float32(eps), hq, hkv, d, 5e5, style)
    for name, got, w in (("q", q, want[0]), ("k", k, want[1])):
        # the sum of squares, its root, the quotient and two products: well below 2^-18
        bound = _rope_bound(w, d, style) + 2.0 ** -18 * np.abs(w)
        assert (np.abs(f64_of(got)[:n] - w) <= bound).all(), name
    _same(f64_of(v)[:n], want[2], "v")
    assert all((f64_of(t)[n:] == 55).all() for t in (q, k, v))
    q2, k2 = torch.empty_like(q), torch.empty_like(k)
    B.ct_qk_norm_rope(*args, q2, k2, None)
    assert np.array_equal(bits_of(q2)[:n], bits_of(q)[:n]) and np.array_equal(bits_of(k2)[:n], bits_of(k)[:n])


@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("d", [64, 128])
def test_norm_of_heads_whose_squares_leave_single_precision(eps, d):
    """Heads of every size that bf16 holds: the norm brings them all to the size of the weights (eps permitting)."""
    hq, hkv = 8, 2
    say(f"qk norm sizes d={d} eps={eps}")
    rng = np.random.default_rng(d)
    x = rng.standard_normal((5, hq + 2 * hkv, d)) * 2.0 ** np.linspace(-120, 124, 12)[None, :, None]
    x = W.f32_to_bf16_bits(x.astype(np.float32))
    w = W.f32_to_bf16_bits((1 + 0.3 * rng.standard_normal(d)).astype(np.float32))
    pos = np.array([0, 1, 77, 4096, 100000], dtype=np.int32)
    q, k, v = (torch.empty((5, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    B.ct_qk_norm_rope(_cfg(hq, hkv, d, 5e5), dev_bf16(x.reshape(5, -1)), dev_i32(pos), 5, dev_bf16(w), dev_bf16(w), eps, q, k, v)
    wf = W.bf16_bits_to_f64(w)
    want = O.qk_norm_rope(W.bf16_bits_to_f64(x).reshape(5, -1), pos, wf, wf, np.float32(eps), hq, hkv, d, 5e5)
    for got, r in ((q, want[0]), (k, want[1])):
        # 2^-133: the step of bf16 below its normal numbers
        assert (np.abs(f64_of(got) - r) <= _rope_bound(r, d, 0) + 2.0 ** -18 * np.abs(r) + 2.0 ** -133).all()
    _same(f64_of(v), want[2], "v")


def test_norm_of_zeros_and_of_what_is_not_finite():
    """A head of zeros stays zero; NaN and infinities stay in their head."""
    hq, hkv, d = 4, 2, 64
    say("qk norm special")
    rng = np.random.default_rng(2)
    x = _bits(rng, 3, (hq + 2 * hkv), d)
    x[0, 1], x[1, 4, 7], x[2, 2, 5] = 0, 0x7fc0, 0x7f80
    one = W.f32_to_bf16_bits(np.ones(d, dtype=np.float32))
    q, k, v = (torch.empty((3, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    B.ct_qk_norm_rope(_cfg(hq, hkv, d), dev_bf16(x.reshape(3, -1)), dev_i32([5, 6, 7]), 3, dev_bf16(one), dev_bf16(one), 1e-6, q, k, v)
    gq, gk = f64_of(q), f64_of(k)
    assert (gq[0, 1] == 0).all() and np.isnan(gk[1, 0]).all() and not np.isfinite(gq[2, 2]).all()
    gq[0, 1] = gk[1, 0] = gq[2, 2] = 1
    assert np.isfinite(gq).all() and np.isfinite(gk).all()


# ---------------------------------------------------------------------------------- together
@pytest.mark.parametrize("hq,hkv,d,bits", [(8, 2, 64, 4), (16, 8, 128, 8)])
def test_tokens_generated_one_after_the_other(hq, hkv, d, bits):
    """Two requests take turns of one and of three tokens: projection, norms and rotation, rows appended to the packed
    cache (values straight out of the projected rows, a padded row left out), attention over all of it.  Each step is
    held to the oracle on what the step before left."""
    say(f"generation heads={hq}/{hkv} d={d} bits={bits}")
    rng = np.random.default_rng(31)
    hidden, o = 256, (hq + 2 * hkv) * d
    cfg = B.make_cfg(hidden, hq, hkv, d, 1e4)
    n_rows, starts, lens = 512, np.array([9, 300]), np.array([200, 37])
    w = dev_bf16(W.f32_to_bf16_bits((rng.standard_normal((o, hidden)) / 16).astype(np.float32)))
    qw, kw = (W.f32_to_bf16_bits((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)) for _ in range(2))
    cache = _cache(cfg, n_rows, bits)
    for s, n in zip(starts, lens):
        _pack(cfg, _bits(rng, n, hkv, d), _bits(rng, n, hkv, d), cache, n_rows, bits, None, int(s))
    for n_new in (1, 3, 1):
        lens = lens + n_new
        n = 2 * n_new
        pos = np.concatenate([np.arange(m - n_new, m) for m in lens])
        rows = np.concatenate([s + np.arange(m - n_new, m) for s, m in zip(starts, lens)])
        x = dev_bf16(_bits(rng, n + 1, hidden, spread=0.1))                   # one row of padding
        qkv = torch.empty((n + 1, o), dtype=torch.bfloat16, device="cuda")
        q, k = (torch.empty((n + 1, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
        out = torch.empty((2, n_new, hq, d), dtype=torch.bfloat16, device="cuda")
        B.ct_linear(x, n + 1, hidden, w, o, None, qkv)
        B.ct_qk_norm_rope(cfg, qkv, dev_i32(np.r_[pos, 0]), n + 1, dev_bf16(qw), dev_bf16(kw), 1e-6, q, k, None)
        before = _read(cfg, cache, n_rows, bits, hkv, d)
        B.ct_pack_kv(cfg, k, hkv * d, qkv[:, (hq + hkv) * d:], o, n + 1, dev_i32(np.r_[rows, -1]), 0, cache, n_rows, bits)
        _attend(cfg, q, 2, n_new, cache, n_rows, bits, starts, lens, 256, out)
        wq, wk, wv = O.qk_norm_rope(f64_of(qkv)[:n], pos, W.bf16_bits_to_f64(qw), W.bf16_bits_to_f64(kw), 1e-6, hq, hkv, d, 1e4)
        for got, want in ((q, wq), (k, wk)):
            assert (np.abs(f64_of(got)[:n] - want) <= _rope_bound(want, d, 0) + 2.0 ** -18 * np.abs(want)).all()
        after = _read(cfg, cache, n_rows, bits, hkv, d)
        for a, b0, new in ((after[0], before[0], f64_of(k)[:n]), (after[1], before[1], wv)):
            want = b0.copy()
            want[rows] = O.packed_values(new, bits)
            _same(a, want, "cache")
        for b in range(2):
            span = slice(starts[b], starts[b] + lens[b])
            _held_to_oracle(f64_of(out)[b], f64_of(q)[b * n_new:(b + 1) * n_new], after[0][span], after[1][span],
                            f"attention, request {b}, {n_new} new")


@pytest.mark.parametrize("hq,hkv,d,bits,style", [(8, 2, 64, 8, 0), (16, 8, 128, 4, 1)])
def test_partial_prefill_from_a_packed_pool(hq, hkv, d, bits, style):
    """Chunks cached in a packed pool make up a context: read back to their new positions without the recompute set's
    rows, the selected rows projected and scattered, their attention over the fused buffers; then the whole context
    goes to a packed cache of the running request, and its next token attends over that."""
    say(f"prefill from a packed pool heads={hq}/{hkv} d={d} bits={bits}")
    rng = np.random.default_rng(41)
    lens, hidden = [70, 33, 128, 1], 128
    cfg = B.make_cfg(hidden, hq, hkv, d, 1e4, style)
    n_ctx, n_rows = sum(lens), 256
    order, at = [2, 0, 3, 1], {}
    k, v = _bits(rng, n_rows, hkv, d, spread=0.0), _bits(rng, n_rows, hkv, d, spread=0.0)      # unit scale, for its bounds
    pool = _cache(cfg, n_rows, bits)
    _pack(cfg, k, v, pool, n_rows, bits)
    row = 5
    for c in order:
        at[c] = row
        row += lens[c]
    rows = np.concatenate([at[c] + np.arange(n) for c, n in enumerate(lens)]).astype(np.int32)
    old = np.concatenate([np.arange(n) for n in lens]).astype(np.int32)
    new = np.arange(n_ctx, dtype=np.int32)
    sel = np.sort(rng.permutation(n_ctx)[:40]).astype(np.int32)
    read = rows.copy()
    read[sel] = -1
    kb, vb = (torch.full((n_ctx, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ct_unpack_kv(cfg, pool, n_rows, bits, dev_i32(read), 0, dev_i32(old), dev_i32(new), n_ctx, kb, vb)
    x = _bits(rng, 40, hidden, spread=0.1)
    wq = W.f32_to_bf16_bits((rng.standard_normal(((hq + 2 * hkv) * d, hidden)) / np.sqrt(hidden)).astype(np.float32))
    q, ks, vs = (torch.empty((40, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    out = torch.empty_like(q)
    ws = torch.empty(max(256, B.ct_workspace_bytes(cfg, n_ctx, 40)), dtype=torch.uint8, device="cuda")
    B.ct_qkv_selected(cfg, dev_bf16(x), None, dev_i32(new[sel]), 40, dev_bf16(wq), None, q, ks, vs)
    B.ct_scatter_kv(cfg, kb, vb, n_ctx, ks, vs, dev_i32(sel), 40)
    B.ct_selected_attention(cfg, q, kb, vb, n_ctx, dev_i32(sel), 40, out, None, ws, ws.numel())
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(t), bits) for t in (k, v))
    want = O.partial_prefill_layer(W.bf16_bits_to_f64(x), W.bf16_bits_to_f64(wq), None, kv[rows], vv[rows], old, new, sel, hq,
                                   hkv, d, 1e4, style)[0]
    assert_close(f64_of(out), want, "selected attention over a packed pool")
    # on with the request
    run_rows = 320
    cache = _cache(cfg, run_rows, bits)
    B.ct_pack_kv(cfg, kb, hkv * d, vb, hkv * d, n_ctx, None, 32, cache, run_rows, bits)
    out1 = torch.empty((1, 1, hq, d), dtype=torch.bfloat16, device="cuda")
    _attend(cfg, q[39:], 1, 1, cache, run_rows, bits, [32], [n_ctx], n_ctx, out1)
    kf, vf = O.packed_values(f64_of(kb), bits), O.packed_values(f64_of(vb), bits)
    _held_to_oracle(f64_of(out1)[0], f64_of(q)[39:], kf, vf, "next token")


def test_captured_and_replayed_with_other_lengths():
    """One decoding step captured into a graph, replayed while the sequences grow and eager calls run between; a second
    graph with a workspace of its own."""
    hq, hkv, d, bits, n_rows, top = 16, 8, 128, 4, 4096, 1500
    say("packed decoding step in a graph")
    rng = np.random.default_rng(51)
    cfg = _cfg(hq, hkv, d)
    starts = dev_i32([5, 2000])
    need = B.ct_packed_attention_workspace_bytes(cfg, 2, 1, top)
    assert need > 0
    one = dev_bf16(W.f32_to_bf16_bits(np.ones(d, dtype=np.float32)))

    class Step:
        def __init__(self):
            self.cache = _cache(cfg, n_rows, bits)
            _pack(cfg, k0, v0, self.cache, n_rows, bits)
            self.qkv = torch.zeros((2, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device="cuda")
            self.pos, self.rows, self.lens = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(3))
            self.q, self.k, self.out = (torch.zeros((2, 1, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hq))
            self.lse = torch.zeros((2, 1, hq), dtype=torch.float32, device="cuda")
            self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")

        def set(self, x, lens):
            self.qkv.copy_(x)
            self.lens.copy_(dev_i32(lens))
            self.pos.copy_(self.lens - 1)
            self.rows.copy_(starts + self.lens - 1)

        def run(self, stream):
            B.ct_qk_norm_rope(cfg, self.qkv, self.pos, 2, one, one, 1e-6, self.q, self.k, None, stream)
            B.ct_pack_kv(cfg, self.k, hkv * d, self.qkv[:, (hq + hkv) * d:], self.qkv.stride(0), 2, self.rows, 0, self.cache, n_rows, bits, stream)
            B.ct_packed_attention(cfg, self.q, 2, 1, self.cache, n_rows, bits, starts, self.lens, top, self.out, self.lse, self.ws, need, stream)

    k0, v0 = _bits(rng, n_rows, hkv, d), _bits(rng, n_rows, hkv, d)
    eager, steps, graphs = Step(), [Step(), Step()], []
    x0 = dev_bf16(_bits(rng, 2, (hq + 2 * hkv) * d))
    for s in steps + [eager]:
        s.set(x0, [1, 1])
        s.run(None)
    torch.cuda.synchronize()
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.run(torch.cuda.current_stream())
        graphs.append(g)
    for i, lens in enumerate([[1, 700], [1499, 3], [1500, 0], [0, 1500], [40, 41]]):
        x = dev_bf16(_bits(rng, 2, (hq + 2 * hkv) * d))
        for s in steps + [eager]:
            s.set(x, lens)
        side = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for g, st in zip(graphs, side):
            with torch.cuda.stream(st):
                g.replay()
        eager.run(None)
        torch.cuda.synchronize()
        for s in steps:
            assert torch.equal(s.out.view(torch.int16), eager.out.view(torch.int16)), f"replay {i}"
            assert torch.equal(s.lse, eager.lse), f"replay {i}"
            assert torch.equal(s.cache, eager.cache), f"replay {i}: cache"


def test_on_a_stream_of_its_own():
    """Work ordered on a side stream alone: the calls must not touch any other stream."""
    hq, hkv, d, bits, n = 32, 8, 128, 8, 2048
    say("packed calls on a side stream")
    g = torch.Generator(device="cuda").manual_seed(4)
    cfg, st = _cfg(hq, hkv, d), torch.cuda.Stream()
    k, v = (torch.randn((n, hkv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((1, 1, hq, d), generator=g, device="cuda").to(torch.bfloat16)
    need = B.ct_packed_attention_workspace_bytes(cfg, 1, 1, n)
    start, length, new = dev_i32([0]), dev_i32([n]), dev_i32(np.arange(n))
    results = []
    for stream in (None, st):
        cache, ws = _cache(cfg, n, bits), torch.empty(need, dtype=torch.uint8, device="cuda")
        out, k2, v2 = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        big = torch.zeros(1 << 28, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(stream) if stream else torch.cuda.stream(torch.cuda.default_stream()):
            for _ in range(8):
                big += 1                                       # keeps the stream busy ahead of the calls
            B.ct_pack_kv(cfg, k, hkv * d, v, hkv * d, n, None, 0, cache, n, bits, stream)
            B.ct_unpack_kv(cfg, cache, n, bits, None, 0, None, new, n, k2, v2, stream)
            B.ct_packed_attention(cfg, q, 1, 1, cache, n, bits, start, length, n, out, None, ws, need, stream)
        if stream:
            stream.synchronize()
        else:
            torch.cuda.synchronize()
        results.append((out.clone(), k2.clone(), v2.clone()))
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
