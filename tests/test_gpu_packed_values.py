"""The values that a packed cache stands for, over all bf16 numbers: rows written and read back bit for bit, and the scales
that the attention reads beside one another, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import ct_oracle as O
from paper_2605_24022_amd import binding as B
from paper_2605_24022_amd import workloads as W
from tests.gpu_util import dev_bf16, dev_i32, f64_of, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available()
    B.load()
    torch.cuda.set_device(0)


MANTISSAS = np.array([0x00, 0x5f, 0x60, 0x61, 0x7f])      # both sides of 1.75, where the scale changes, and the ends


def _there_and_back(groups, d, bits):
    """Groups [n, 32] of bf16 patterns as the K rows of one head, and in the opposite order as its V rows."""
    per_row = d // 32
    n = -(-groups.shape[0] // (32 * per_row)) * 32
    x = np.zeros((n * per_row, 32), dtype=np.uint16)
    x[: groups.shape[0]] = groups
    x = x.reshape(n, 1, d)
    cfg = B.make_cfg(64 * d, 1, 1, d, 1e4, 0, 0.0)
    cache = torch.full((B.ct_packed_kv_bytes(cfg, n, bits),), 0xff, dtype=torch.uint8, device="cuda")
    B.ct_pack_kv(cfg, dev_bf16(x), d, dev_bf16(x[::-1]), d, n, None, 0, cache, n, bits)
    k, v = (torch.full((n, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ct_unpack_kv(cfg, cache, n, bits, None, 0, None, None, n, k, v)
    want = O.packed_values(W.bf16_bits_to_f64(x), bits)
    for name, got in (("K", f64_of(k)), ("V", f64_of(v)[::-1])):
        bad = got != want
        assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} differ, first {got[bad][0]} for {want[bad][0]}"


def _in_groups(tops, elements):
    """31 elements a group behind its largest one; elements above it become it."""
    e = np.concatenate([elements, elements[: -elements.size % 31]]).reshape(-1, 31)
    out = np.empty((tops.size, e.shape[0], 32), dtype=np.uint16)
    out[:, :, 0] = tops[:, None]
    out[:, :, 1:] = np.where((e & 0x7fff)[None] <= tops[:, None, None], e[None], tops[:, None, None])
    return out.reshape(-1, 32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("exponents", [(0, 8, 9, 10), (12, 100, 127, 128), (200, 252, 253, 254)])
def test_all_finite_numbers_beside_borders_of_some_scales(d, bits, exponents):
    say(f"packed values, all finite ones, d={d} bits={bits} exponents={exponents}")
    every = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    every = every[(every & 0x7f80) != 0x7f80]
    tops = ((np.array(exponents)[:, None] << 7) | MANTISSAS[None]).ravel().astype(np.uint16)
    _there_and_back(_in_groups(tops, every), d, bits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
def test_numbers_that_count_beside_borders_of_all_scales(d, bits):
    """Every exponent of the largest magnitude, both sides of the border, with all numbers down to those that become zero."""
    reach = 6 if bits == 4 else 19
    say(f"packed values, all scales, d={d} bits={bits}")
    groups = []
    for exp in range(255):
        below = np.arange(max(exp - reach, 0) << 7, (exp + 1) << 7)
        below = np.concatenate([below, below | 0x8000]).astype(np.uint16)
        groups.append(_in_groups(((exp << 7) | MANTISSAS).astype(np.uint16), below))
    _there_and_back(np.concatenate(groups), d, bits)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
def test_scales_beside_any_others(d, bits):
    """The attention takes scales out of words that hold their neighbours'.  One key of a sequence gets all the weight: the
    log-sum-exp is its score, one element of q times one of k, the output its V row, bit for bit.  Its scales go through
    all bytes and places while those beside it are anything.

    The scores are 400 for this key and 0 for the others, whose weights are zero; the output is p v / p with p within 2^-16
    of 1, and v a bf16 number; the log-sum-exp is off by a few fp32 roundings of 400 and of 400 log2 e."""
    hkv, n_seq, length = 2, 512, 64
    emax = 2 if bits == 4 else 8
    first, last = 10, 254 - emax                       # scale bytes
    say(f"packed scales beside others d={d} bits={bits}")
    rng = np.random.default_rng([d, bits])
    cfg = B.make_cfg(hkv * d, hkv, hkv, d, 1e4, 0, 1.0)
    n_rows, groups = n_seq * length, d // 32

    def power(byte):                                   # pattern of the power of two that makes it the group's scale
        return ((byte + emax) << 7).astype(np.uint16)

    # K: an element of each group sets its scale (element 0, which q does not look at); the key's own group has element 5
    k = np.zeros((n_seq, length, hkv, groups, 32), dtype=np.uint16)
    k[..., 0] = power(rng.integers(first, last + 1, k.shape[:-1]))
    v = rng.integers(0, 1 << 16, (n_seq, length, hkv, groups, 32)).astype(np.uint16)
    byte = rng.integers(first, last + 1, v.shape[:-1])
    byte[..., :] = np.where(rng.random(byte.shape) < 0.1, first + rng.integers(0, 2, byte.shape), byte)
    top = power(byte)
    v = np.where((v & 0x7fff) < (top[..., None] | 0x60), v, (v & 0x807f) | top[..., None])      # none above the scale's limit ...
    v = np.where((v & 0x7fff) <= (top[..., None] | 0x60), v, top[..., None])
    v[..., 7] = top                                                                             # ... and one that needs it
    q = np.zeros((n_seq, hkv, groups, 32), dtype=np.uint16)
    s, g = np.meshgrid(np.arange(n_seq), np.arange(hkv), indexing="ij")
    row, group = s % 32, (s // 32 + g) % groups
    own = first + (s * hkv + g) * 7 % (last + 1 - first)                                        # 7 is prime to 243 and 237
    k[s, row, g, group, 0] = 0
    k[s, row, g, group, 5] = power(own)
    exp = 127 + 8 - (own + emax - 127)                                                          # 400 = 1.5625 * 2^8
    q[s, g, group, 5] = (exp << 7) | 0x48
    assert exp.min() > 0 and exp.max() < 255
    vb = first + (s * hkv + g + 100) * 5 % (last + 1 - first)
    for i in range(groups):
        v[s, row, g, i, 7] = power(vb)
        v[s, row, g, i] = np.where((v[s, row, g, i] & 0x7fff) <= power(vb)[..., None], v[s, row, g, i], power(vb)[..., None])
    k, v = k.reshape(n_rows, hkv, d), v.reshape(n_rows, hkv, d)
    cache = torch.full((B.ct_packed_kv_bytes(cfg, n_rows, bits),), 0xff, dtype=torch.uint8, device="cuda")
    B.ct_pack_kv(cfg, dev_bf16(k), hkv * d, dev_bf16(v), hkv * d, n_rows, None, 0, cache, n_rows, bits)
    out = torch.full((n_seq, 1, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_seq, 1, hkv), float("nan"), device="cuda")
    assert B.ct_packed_attention_workspace_bytes(cfg, n_seq, 1, length) == 0
    B.ct_packed_attention(cfg, dev_bf16(q.reshape(n_seq, 1, hkv, d)), n_seq, 1, cache, n_rows, bits, dev_i32(np.arange(n_seq) * length),
                          dev_i32(np.full(n_seq, length)), length, out, lse, None, 0)
    got_lse = lse.cpu().numpy().astype(np.float64)[:, 0]
    off = np.abs(got_lse - 400) > 2.0 ** -21 * 400
    assert not off.any() and not np.isnan(got_lse).any(), f"K scale bytes {sorted(set(own[off].tolist()))[:8]}: {got_lse[off][:4]}"
    want = O.packed_values(W.bf16_bits_to_f64(v.reshape(n_seq, length, hkv, d)[s, row, g]), bits)
    assert np.isfinite(want).all() and set(vb.ravel().tolist()) == set(range(first, last + 1))
    got = f64_of(out)[:, 0]
    bad = got != want
    assert not bad.any(), f"V: {bad.sum()} of {bad.size} differ, first {got[bad][0]} for {want[bad][0]}"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("power", [8, 16, 24, 28])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(d, bits, power, sign):
    """Scores of about 2^power of either sign: the key ahead of the others by half of that gets all the weight, its V row
    comes out bit for bit, and the log-sum-exp is its score, off by a few fp32 roundings of it and of it times log2 e."""
    hkv, n_seq, length = 2, 96, 200
    say(f"packed scores of 2^{power} d={d} bits={bits} sign={sign}")
    rng = np.random.default_rng([d, bits, power])
    cfg = B.make_cfg(hkv * d, hkv, hkv, d, 1e4, 0, 1.0)
    n_rows = n_seq * length // 32 * 32 + 32
    ahead, behind = (1.5, 1.0) if sign > 0 else (-1.0, -1.5)        # exact in both formats, alone in their group
    k = np.zeros((n_rows, hkv, d))
    k[..., 37] = behind
    best = rng.integers(0, length, (n_seq, hkv))
    start = np.arange(n_seq) * length
    for h in range(hkv):
        k[start + best[:, h], h, 37] = ahead
    q = np.zeros((n_seq, 1, hkv, d))
    q[..., 37] = 2.0 ** power
    v = rng.standard_normal((n_rows, hkv, d))
    kb, vb, qb = (W.f32_to_bf16_bits(x.astype(np.float32)) for x in (k, v, q))
    cache = torch.full((B.ct_packed_kv_bytes(cfg, n_rows, bits),), 0xff, dtype=torch.uint8, device="cuda")
    B.ct_pack_kv(cfg, dev_bf16(kb), hkv * d, dev_bf16(vb), hkv * d, n_rows, None, 0, cache, n_rows, bits)
    out = torch.full((n_seq, 1, hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_seq, 1, hkv), float("nan"), device="cuda")
    B.ct_packed_attention(cfg, dev_bf16(qb), n_seq, 1, cache, n_rows, bits, dev_i32(start), dev_i32(np.full(n_seq, length)), length, out,
                          lse, None, 0)
    values = O.packed_values(W.bf16_bits_to_f64(vb), bits)
    want = np.stack([values[start + best[:, h], h] for h in range(hkv)], 1)
    assert np.array_equal(f64_of(out)[:, 0], want)
    score = ahead * 2.0 ** power
    assert (np.abs(lse.cpu().numpy().astype(np.float64) - score) <= 2.0 ** -21 * abs(score)).all()
