"""The scales that the attention over packed caches reads beside one another, against the oracle."""
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
