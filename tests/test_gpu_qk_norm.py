"""Norms of queries and keys over the whole range of weights, against the oracle in 64 bits."""
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


@pytest.mark.parametrize("d,style", [(64, 0), (64, 1), (128, 0), (128, 1)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_weights_of_every_size_beside_heads_of_every_size(d, style, eps):
    """A normed element is of the size of its weight whatever the head's: no product on the way may leave fp32 where the
    result does not.  One weight size per call, 2^-110 to 2^120; a head for each of twelve sizes, 2^-120 to 2^120."""
    hq, hkv, n = 8, 4, 3
    rng = np.random.default_rng([d, style])
    x = rng.standard_normal((n, hq + 2 * hkv, d))
    x[:, :hq + hkv] *= 2.0 ** np.linspace(-120, 120, hq + hkv)[None, :, None]
    x = W.f32_to_bf16_bits(x.astype(np.float32)).reshape(n, -1)
    pos = np.array([0, 77, 100000], dtype=np.int32)
    cfg = B.make_cfg(hq * d, hq, hkv, d, 5e5, style, 0.0)
    for e in (-110, -90, -60, -20, 0, 20, 60, 90, 120):
        say(f"qk norm weights d={d} style={style} eps={eps} 2^{e}")
        qw, kw = (W.f32_to_bf16_bits(((1 + 0.3 * rng.standard_normal(d)) * 2.0 ** e).astype(np.float32)) for _ in range(2))
        q, k = (torch.full((n, h, d), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
        B.ct_qk_norm_rope(cfg, dev_bf16(x), dev_i32(pos), n, dev_bf16(qw), dev_bf16(kw), eps, q, k, None)
        want = O.qk_norm_rope(W.bf16_bits_to_f64(x), pos, W.bf16_bits_to_f64(qw), W.bf16_bits_to_f64(kw), np.float32(eps), hq, hkv, d,
                              5e5, style)
        for name, got, r in (("q", f64_of(q), want[0]), ("k", f64_of(k), want[1])):
            a = np.abs(r)
            pair = np.concatenate([a[..., : d // 2] + a[..., d // 2:]] * 2, -1) if style == 0 else np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1)
            # the result's rounding; sine and cosine are good to 2^-19.5 together and |a| + |b| of a rotated pair is at least
            # 0.7 of the unrotated one's: 2^-18; a sum of up to 128 squares, root, quotient and two products: below 2^-17;
            # 2^-133: the step of bf16 below its normal numbers
            bound = 2.0 ** -8 * a + (2.0 ** -18 + 2.0 ** -17) * pair + 2.0 ** -133
            bad = ~(np.abs(got - r) <= bound)
            assert not bad.any(), f"{name}, weights 2^{e}: {bad.sum()} elements off, heads {sorted(set(np.argwhere(bad)[:, 1]))}"


def test_what_is_not_finite_stays_in_its_place():
    """An infinite element makes a NaN of its rotation pair and zeros of the rest of its head; an infinite weight makes
    infinities of its pair."""
    hq, hkv, d = 2, 1, 64
    say("qk norm infinities")
    rng = np.random.default_rng(3)
    x = W.f32_to_bf16_bits(rng.standard_normal((1, hq + 2 * hkv, d)).astype(np.float32))
    x[0, 0, 5] = 0x7f80
    one = W.f32_to_bf16_bits(np.ones(d, dtype=np.float32))
    inf = one.copy()
    inf[9] = 0x7f80
    q, k = (torch.empty((1, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv))
    B.ct_qk_norm_rope(B.make_cfg(hq * d, hq, hkv, d, 1e4, 0, 0.0), dev_bf16(x.reshape(1, -1)), dev_i32([3]), 1, dev_bf16(one), dev_bf16(inf), 1e-6,
                      q, k, None)
    gq, gk = f64_of(q)[0], f64_of(k)[0]
    assert np.isnan(gq[0, [5, 5 + d // 2]]).all()
    assert (np.delete(gq[0], [5, 5 + d // 2]) == 0).all() and np.isfinite(gq[1]).all()
    assert not np.isfinite(gk[0, [9, 9 + d // 2]]).any() and np.isfinite(np.delete(gk[0], [9, 9 + d // 2])).all()
