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
from tests.gpu_util import bits_of, dev_bf16, dev_i32, f64_of, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available()
    B.load()
    torch.cuda.set_device(0)


def _rows(rng, *shape):
    return W.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def _definition(q, k, v, scale):
    """One sequence: outputs [n_new, Hq, D], log-sum-exp, and how far from them the kernel may be."""
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
            slack = (p * e) @ (np.abs(vg) + np.abs(o)) + (2.0 ** -16 + 2.0 ** -18) * (p @ np.abs(vg))
            out[t, h], off[t, h] = o, 2.0 ** -8 * (np.abs(o) + slack) + slack
            lse[t, h] = s.max() + np.log(w.sum())
            lse_off[t, h] = p @ e + 2.0 ** -18 + 2.0 ** -22 * abs(lse[t, h])
    return out, off, lse, lse_off


def _check(hq, hkv, d, bits, n_new, lens, starts, n_rows, max_len=None, parts=None):
    """The call against the definition; rows outside the sequences read as NaN.  parts: into how many the key range of
    max_len rows has to be divided."""
    max_len = max(lens) if max_len is None else max_len
    say(f"packed attention heads={hq}/{hkv} d={d} bits={bits} n_new={n_new} lens={lens[:8]} max_len={max_len} rows={n_rows} parts={parts}")
    rng = np.random.default_rng([hq, hkv, d, bits, n_new, len(lens)])
    cfg = B.make_cfg(hq * d, hq, hkv, d, 1e4, 0, 0.0)
    n_seq = len(lens)
    need = B.ct_packed_attention_workspace_bytes(cfg, n_seq, n_new, max_len)
    got_parts = max(1, need // (n_seq * hq * n_new * (d + 2) * 4))
    assert parts is None or got_parts == parts, f"divided into {got_parts} parts"
    cache = torch.full((B.ct_packed_kv_bytes(cfg, n_rows, bits),), 0xff, dtype=torch.uint8, device="cuda")
    k, v, q = _rows(rng, n_rows, hkv, d), _rows(rng, n_rows, hkv, d), _rows(rng, n_seq, n_new, hq, d)
    inside = np.zeros(n_rows, dtype=bool)
    for s, n in zip(starts, lens):
        inside[s:s + n] = True
    rows = np.flatnonzero(inside).astype(np.int32)
    kd, vd = dev_bf16(k[rows]), dev_bf16(v[rows])
    B.ct_pack_kv(cfg, kd, hkv * d, vd, hkv * d, rows.size, dev_i32(rows), 0, cache, n_rows, bits)
    out = torch.full((n_seq, n_new, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_seq, n_new, hq), float("nan"), dtype=torch.float32, device="cuda")
    ws = torch.full((max(need, 256),), 0xff, dtype=torch.uint8, device="cuda")
    B.ct_packed_attention(cfg, dev_bf16(q), n_seq, n_new, cache, n_rows, bits, dev_i32(starts), dev_i32(lens), max_len, out, lse, ws, need)
    got, got_lse = f64_of(out), lse.cpu().numpy().astype(np.float64)
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(x), bits) for x in (k, v))
    qv = W.bf16_bits_to_f64(q)
    for b, (s, n) in enumerate(zip(starts, lens)):
        want, off, want_lse, lse_off = _definition(qv[b], kv[s:s + n], vv[s:s + n], d ** -0.5)
        beyond = np.abs(got[b] - want) - off
        assert not (beyond > 0).any() and not np.isnan(got[b]).any(), \
            f"sequence {b}: {(beyond > 0).sum()} of {beyond.size} outputs beyond their bound, by up to {np.nanmax(beyond / np.maximum(off, 1e-30))} of it"
        fin = np.isfinite(want_lse)
        assert np.array_equal(got_lse[b][~fin], want_lse[~fin])
        assert (np.abs(got_lse[b] - want_lse)[fin] <= lse_off[fin]).all(), f"sequence {b}: log-sum-exp"


# ---------------------------------------------------------------------------------- precision
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128), (16, 16, 64), (8, 1, 128)])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_new", [1, 5])
def test_outputs_are_off_by_their_own_rounding_alone(hq, hkv, d, bits, n_new):
    """Weights enter the product with the values in more than the bits of one bf16 number."""
    _check(hq, hkv, d, bits, n_new, [5, 64, 200, 700], [3, 10, 80, 300], 1024)
