"""Attention over packed caches, every kernel of it by itself, against the definition in 64 bits.

Bounds.  With p_j the softmax weights and o the output, an output moves by sum_j p_j e_j (v_j - o) where the weight of key j is
off by e_j of itself, and by sum_j p_j r_j v_j where it enters the product with v off by r_j.  e_j: a score of D exact products
added in fp32 is off by D 2^-24 sum |q k| scale; the scale and log2 e in fp32, their products with the score and with the
maximum, 2^-22 of either; the exponential 2^-20.  r_j: a sum of two bf16 numbers, 2^-16.  fp32 sums over up to 2^16 keys: 2^-18
of sum p |v| (a wave adds 32 keys at a time, waves and parts add theirs up).  The rounding of the result: 2^-8 of it."""
import numpy as np
import pytest
import torch

from oracle import ct_oracle as O
from paper_2605_24022_amd import binding as B
from paper_2605_24022_amd import workloads as W
from tests.gpu_util import dev_bf16, dev_i32, f64_of, say
from tests.test_gpu_packed import _check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available()
    B.load()
    torch.cuda.set_device(0)


def _rows(rng, *shape):
    return W.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def _definition(q, k, v, scale, floor=0.0):
    """One sequence: outputs [n_new, Hq, D], log-sum-exp, and how far from them the kernel may be (floor: see where it is
    given)."""
    n_new, hq, d = q.shape
    n, hkv, _ = k.shape
    out, off = np.zeros((n_new, hq, d)), np.zeros((n_new, hq, d))
    lse, lse_off = np.full((n_new, hq), -np.inf), np.zeros((n_new, hq))
    for t in range(n_new):
        seen = n - n_new + t + 1
        if seen <= 0:
            continue
        for h in range(hq):
            kg, vg = k[:seen, h // (hq // hkv)], v[:seen, h // (hq // hkv)]
            s = kg @ q[t, h] * scale
            w = np.exp(s - s.max())
            p = w / w.sum()
            o = p @ vg
            e = d * 2.0 ** -24 * (np.abs(kg) @ np.abs(q[t, h])) * scale + 2.0 ** -22 * (np.abs(s) + abs(s.max())) + 2.0 ** -20
            slack = (p * e) @ (np.abs(vg) + np.abs(o)) + (2.0 ** -16 + 2.0 ** -18) * (p @ np.abs(vg)) + floor * seen / w.sum()
            out[t, h], off[t, h] = o, 2.0 ** -8 * (np.abs(o) + slack) + slack
            lse[t, h] = s.max() + np.log(w.sum())
            lse_off[t, h] = p @ e + 2.0 ** -18 + 2.0 ** -22 * abs(lse[t, h])
    return out, off, lse, lse_off


def _check(hq, hkv, d, bits, n_new, lens, starts, n_rows, max_len=None, divided=None, by_length=None, streamed=None,
           values=_rows, queries=_rows, floor=0.0):
    """The call against the definition; rows outside the sequences read as NaN.  What the case is there for is held to the
    rules of the host: `divided`, the key range of max_len rows (which the workspace shows); `by_length`, whole sequences
    on more than 256 workgroups; `streamed`, 8-bit codes on one workgroup for all columns, rows enough for all sequences."""
    max_len = max(lens) if max_len is None else max_len
    say(f"packed attention heads={hq}/{hkv} d={d} bits={bits} n_new={n_new} lens={lens[:8]} max_len={max_len} rows={n_rows}")
    rng = np.random.default_rng([hq, hkv, d, bits, n_new, len(lens)])
    cfg = B.make_cfg(hq * d, hq, hkv, d, 1e4, 0, 0.0)
    n_seq, cols = len(lens), n_new * hq // hkv
    need = B.ct_packed_attention_workspace_bytes(cfg, n_seq, n_new, max_len)
    if divided is not None:
        assert (need > 0) == divided, f"workspace of {need} bytes"
    if by_length is not None:
        col_blocks = 1 if cols <= 16 else -(-cols // 32)
        assert (need == 0 and n_seq * hkv * col_blocks > 256 and n_seq <= 256 and max_len > 2048) == by_length
    if streamed is not None:
        assert (bits == 4 or (cols <= 32 and n_seq * max_len <= n_rows)) == streamed
    cache = torch.full((B.ct_packed_kv_bytes(cfg, n_rows, bits),), 0xff, dtype=torch.uint8, device="cuda")
    rows = np.unique(np.concatenate([np.arange(s, s + n) for s, n in zip(starts, lens)])).astype(np.int32)
    k, v, q = _rows(rng, rows.size, hkv, d), values(rng, rows.size, hkv, d), queries(rng, n_seq, n_new, hq, d)
    kd, vd = dev_bf16(k), dev_bf16(v)
    B.ct_pack_kv(cfg, kd, hkv * d, vd, hkv * d, rows.size, dev_i32(rows), 0, cache, n_rows, bits)
    out = torch.full((n_seq, n_new, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_seq, n_new, hq), float("nan"), dtype=torch.float32, device="cuda")
    ws = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device="cuda")
    B.ct_packed_attention(cfg, dev_bf16(q), n_seq, n_new, cache, n_rows, bits, dev_i32(starts), dev_i32(lens), max_len, out, lse, ws, need)
    got, got_lse = f64_of(out), lse.cpu().numpy().astype(np.float64)
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(x), bits) for x in (k, v))
    qv = W.bf16_bits_to_f64(q)
    for b, (s, n) in enumerate(zip(starts, lens)):
        at = np.searchsorted(rows, s)
        want, off, want_lse, lse_off = _definition(qv[b], kv[at:at + n], vv[at:at + n], d ** -0.5, floor)
        beyond = np.abs(got[b] - want) - off
        assert not (beyond > 0).any() and not np.isnan(got[b]).any(), \
            f"sequence {b}: {(beyond > 0).sum()} of {beyond.size} outputs beyond their bound, by up to {np.nanmax(beyond / np.maximum(off, 1e-30))} of it"
        fin = np.isfinite(want_lse)
        assert np.array_equal(got_lse[b][~fin], want_lse[~fin])
        assert (np.abs(got_lse[b][fin] - want_lse[fin]) <= lse_off[fin]).all(), f"sequence {b}: log-sum-exp"


# ---------------------------------------------------------------------------------- precision
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128), (16, 16, 64), (8, 1, 128)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_new", [1, 5])
def test_outputs_are_off_by_their_own_rounding_alone(hq, hkv, d, bits, n_new):
    """Weights enter the product with the values in more than the bits of one bf16 number."""
    _check(hq, hkv, d, bits, n_new, [5, 64, 200, 700], [3, 10, 80, 300], 1024)


# ---------------------------------------------------------------------------------- every kernel and plan
HEADS = {64: (8, 2), 128: (32, 8)}      # four columns of queries per new token


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits,n_new,room", [
    (4, 1, 0), (4, 5, 0), (4, 12, 0),                    # 16 columns a workgroup, 32, and two workgroups of them
    (8, 1, 0), (8, 5, 0), (8, 1, 1), (8, 5, 1),          # codes through the caches, and past them
    (8, 12, 1)])                                         # (through them: two workgroups read the same codes)
@pytest.mark.parametrize("long", [False, True])
def test_every_kernel_whole_and_divided(d, bits, n_new, room, long):
    """Each pair of head size and bits, 16 and 32 columns, codes read through the caches or past them, the key range
    whole and in parts."""
    hq, hkv = HEADS[d]
    lens = [4900, 70, 333] if long else [400, 33, 70]
    starts = [7, 4910, 4990] if long else [7, 408, 450]
    top = max(lens)
    n_rows = ((3 * top if room else 0) + starts[-1] + lens[-1] + 31) // 32 * 32
    _check(hq, hkv, d, bits, n_new, lens, starts, n_rows, divided=long, streamed=bits == 4 or (room == 1 and n_new < 12))


@pytest.mark.parametrize("d,hq,hkv", [(64, 16, 16), (128, 32, 8)])
@pytest.mark.parametrize("bits,n_new,n_seq,room", [
    (4, 1, 33, 0), (8, 1, 33, 0), (8, 1, 33, 1), (8, 1, 70, 0), (4, 20, 33, 0), (8, 5, 33, 0), (8, 5, 33, 1), (4, 12, 33, 0), (8, 20, 33, 1), (8, 36, 33, 0)])
def test_every_kernel_in_the_order_of_lengths(d, hq, hkv, bits, n_new, n_seq, room):
    """Whole sequences taken by length, with one workgroup for their columns and with several."""
    rng = np.random.default_rng([d, n_seq])
    lens = rng.choice([0, 1, 31, 32, 33, 64, 70], n_seq)
    lens[[1, n_seq // 2, n_seq - 1]] = 2049, 2100, 300
    lens = lens.tolist()
    starts = (3 + np.concatenate([[0], np.cumsum(lens)[:-1]])).tolist()
    n_rows = (max(n_seq * 2100 if room else 0, starts[-1] + lens[-1]) + 31) // 32 * 32
    cols = n_new * hq // hkv
    _check(hq, hkv, d, bits, n_new, lens, starts, n_rows, by_length=True, streamed=bits == 4 or (room == 1 and cols <= 32))


def test_more_than_one_part_each_way():
    """Sequences of a divided batch that end in their first part, on its border and beyond; one of no rows."""
    _check(16, 8, 128, 8, 3, [0, 1, 127, 128, 129, 160, 2500], [0, 5, 6, 140, 270, 400, 561], 3200, max_len=3100, divided=True)


def test_no_rows_at_all():
    """A bound of zero: zeros and minus infinity for everybody, whatever the lengths say."""
    hq, hkv, d = 8, 2, 64
    say("packed attention max_len=0")
    cfg = B.make_cfg(hq * d, hq, hkv, d, 1e4, 0, 0.0)
    cache = torch.full((B.ct_packed_kv_bytes(cfg, 64, 4),), 0xff, dtype=torch.uint8, device="cuda")
    q = dev_bf16(_rows(np.random.default_rng(1), 3, 2, hq, d))
    out, lse = torch.full_like(q, float("nan")), torch.full((3, 2, hq), float("nan"), device="cuda")
    B.ct_packed_attention(cfg, q, 3, 2, cache, 64, 4, dev_i32([0, 5, 60]), dev_i32([0, 7, 4]), 0, out, lse, None, 0)
    assert (f64_of(out) == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_new", [6, 9])
@pytest.mark.parametrize("bad", [0xff80, 0x7fc0])
def test_infinities_and_nan_among_many_columns(hq, hkv, d, bits, n_new, bad):
    """NaN for the new tokens that see it and for no other, with 32 columns a workgroup and with two workgroups of them."""
    def edit(k, v):
        v[16 + 299, 0, 33] = bad          # the last but one token of sequence 0
        v[16 + 300 - 7, 1, 5] = bad       # the last but seven
        k[400 + 69, 0, 1] = bad           # the last but one of sequence 1
        k[400 + 62, 1, 1] = bad           # the last but eight
        v[600 + 3, 1, 40] = bad           # an early row of sequence 2: everybody sees it
        v[15], k[15], v[397], k[396] = bad, bad, bad, bad
    _check_attention(hq, hkv, d, bits, n_new, [301, 71, 50, 3], [16, 400, 600, 394], 704, edit=edit)


# ---------------------------------------------------------------------------------- values at the ends of the range
def _of_exponents(lo, hi):
    """bf16 patterns of any sign and mantissa up to 1.75, exponents lo to hi."""
    def rows(rng, *shape):
        return (rng.integers(0, 2, shape) << 15 | rng.integers(lo, hi + 1, shape) << 7 | rng.integers(0, 0x61, shape)).astype(np.uint16)
    return rows


@pytest.mark.parametrize("hq,hkv,d,n_new", [(8, 2, 64, 1), (32, 8, 128, 1), (32, 8, 128, 5)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("lens", [[700, 33, 1], [5000, 70]])
def test_sums_of_the_largest_values_stay_finite(hq, hkv, d, n_new, bits, lens):
    """Values from 2^126 to 1.75 * 2^127: their average is one of them, their sum is not in fp32.  (A weight of zero for what
    another wave or part has summed up silences a sum, but not an infinity.)"""
    starts = [5, 5 + lens[0], 5 + sum(lens[:2])][:len(lens)]
    _check(hq, hkv, d, bits, n_new, lens, starts, 5120, values=_of_exponents(253, 254))


@pytest.mark.parametrize("hq,hkv,d,n_new", [(8, 2, 64, 1), (32, 8, 128, 5)])
@pytest.mark.parametrize("bits", [4, 8])
def test_the_smallest_values_keep_their_bits(hq, hkv, d, n_new, bits):
    """Values from 2^-126 up.  floor: products and sums are held as 2^-23 of themselves in steps of 2^-149 and off by less
    than one of them, at most three a row (two products, one sum), over a sum of weights of sum_j w_j or more."""
    _check(hq, hkv, d, bits, n_new, [300, 33, 1], [5, 305, 338], 352, values=_of_exponents(1, 18),
           queries=lambda rng, *shape: W.f32_to_bf16_bits((0.05 * rng.standard_normal(shape)).astype(np.float32)), floor=3 * 2.0 ** (23 - 149))
