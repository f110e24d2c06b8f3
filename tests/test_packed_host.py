"""Packed caches and per-head norms without a GPU: the oracle's values against definitions written apart from it, sizes
of caches and workspaces, and what the entry points refuse before any HIP call."""
import numpy as np
import pytest
import torch

from oracle import ct_oracle as O
from paper_2605_24022_amd import binding as B
from paper_2605_24022_amd import workloads as W

FAKE = 0x10000


def _cfg(**kw):
    base = dict(hidden=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, rope_theta=5e5)
    base.update(kw)
    return B.make_cfg(**base)


def _status(fn, *args, **kw):
    with pytest.raises(B.CacheTuneError) as ei:
        fn(*args, **kw)
    assert ei.value.message
    return ei.value.status


# ---------------------------------------------------------------------------------- the oracle's pins
def test_code_values_are_those_of_the_element_formats():
    """e2m1 by hand; e4m3 as torch's type of that name decodes every code."""
    assert O.packed_code_values(4).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.packed_code_values(8), want)


def test_values_by_hand():
    x = np.zeros(32)
    x[:9] = [7, 5, 2.5, 3.5, 0.25, 0.75, -1.25, -6.5, 0.2]     # scale 1; 5 and 2.5 tie to the even code, 7 to the largest value
    assert O.packed_values(x, 4)[:9].tolist() == [6, 4, 2, 4, 0, 1, -1, -6, 0]
    x[0] = 7.03125                                              # above 7: scale 2
    assert O.packed_values(x, 4)[:9].tolist() == [8, 4, 2, 4, 0, 1, -1, -6, 0]
    x[:4] = [448, 18.5, 17, 2 ** -10]                           # scale 1; ties to even; below half the smallest step
    assert O.packed_values(x, 8)[:4].tolist() == [448, 18, 16, 0]
    assert np.isnan(O.packed_values(np.r_[x[:31], np.inf], 8)).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_values_are_the_nearest_and_stay(bits):
    """Every element within half a step of itself (a step of the codes at its magnitude), values in a cache come back as
    they are, and a power of two or a sign ahead of the cache comes out of it unchanged."""
    rng = np.random.default_rng(5)
    x = W.bf16_bits_to_f64(W.f32_to_bf16_bits((rng.standard_normal((40, 64)) * np.exp(rng.standard_normal((40, 1)) * 4)).astype(np.float32)))
    y = O.packed_values(x, bits)
    top = np.abs(x.reshape(40, 2, 32)).max(-1, keepdims=True)
    m, e = np.frexp(top / (1.75 * (4 if bits == 4 else 256)))
    scale = np.ldexp(1.0, np.where(m == 0.5, e - 1, e))
    a = np.abs(x.reshape(40, 2, 32)) / scale
    _, p = np.frexp(a)
    step = np.ldexp(1.0, np.maximum(p - 1, 0 if bits == 4 else -6) - (1 if bits == 4 else 3))
    assert (np.abs(y.reshape(40, 2, 32) / scale - np.sign(x.reshape(40, 2, 32)) * a) <= step / 2).all()
    assert np.array_equal(O.packed_values(y, bits), y)
    assert np.array_equal(O.packed_values(-8 * x, bits), -8 * y)


def test_attention_of_all_tokens_is_causal_attention():
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((9, 4, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    out, lse, _ = O.packed_attention(q, k, v)
    want, want_lse = O.selected_attention(q, k, v, np.arange(9))
    assert np.abs(out - want).max() < 1e-13 and np.abs(lse - want_lse).max() < 1e-13
    out, lse, _ = O.packed_attention(q, k[:2], v[:2])             # more new tokens than the sequence has
    assert (out[:7] == 0).all() and (lse[:7] == -np.inf).all()
    assert np.allclose(out[7], np.repeat(v[0], 2, axis=0)) and np.isfinite(lse[7:]).all()


def test_norm_then_rope():
    """Unit weights and no rotation: rows of root mean square 1; the norm commutes with the rotation for equal weights."""
    rng = np.random.default_rng(7)
    x = rng.standard_normal((3, (4 + 2 * 2) * 64))
    q, k, v = O.qk_norm_rope(x, [0, 0, 0], np.ones(64), np.full(64, 2.0), 0.0, 4, 2, 64, 1e4)
    assert np.allclose((q ** 2).mean(-1), 1) and np.allclose((k ** 2).mean(-1), 4)
    assert np.array_equal(v.reshape(3, -1), x[:, 6 * 64:])
    q2, _, _ = O.qk_norm_rope(x, [5, 6, 7], np.ones(64), np.ones(64), 0.0, 4, 2, 64, 1e4, O.INTERLEAVED)
    assert np.allclose(q2, O.rmsnorm(O.rotate(x.reshape(3, 8, 64)[:, :4], [5, 6, 7], 1e4, O.INTERLEAVED), np.ones(64), 0.0))


# ---------------------------------------------------------------------------------- sizes
def test_cache_bytes():
    for d, hkv, bits in [(128, 8, 4), (128, 8, 8), (64, 2, 4), (64, 16, 8)]:
        c = _cfg(n_q_heads=hkv, n_kv_heads=hkv, head_dim=d)
        for n in (32, 4096):
            assert B.ct_packed_kv_bytes(c, n, bits) == 2 * n * hkv * (d * bits // 8 + d // 32)
    c = _cfg()
    for bad in [(0, 4), (-32, 4), (33, 4), (64, 5), (64, 16)]:
        assert B.ct_packed_kv_bytes(c, *bad) == 0
    assert B.ct_packed_kv_bytes(_cfg(head_dim=96), 64, 4) == 0
    assert B.ct_packed_kv_bytes(c, 0x7fffffe0, 8) == 0x7fffffe0 * 2 * 8 * 132


def test_workspace_bytes():
    c = _cfg()
    assert B.ct_packed_attention_workspace_bytes(c, 1, 1, 64) == 0              # one part
    assert B.ct_packed_attention_workspace_bytes(c, 0, 1, 4096) == 0
    row = 8 * 4 * 130 * 4                                                       # fp32 O, m, l of 8 heads x 4 columns
    need = B.ct_packed_attention_workspace_bytes(c, 1, 1, 32768)
    assert need > row and need % row == 0
    assert B.ct_packed_attention_workspace_bytes(c, 1, 3, 32768) % (3 * row) == 0
    for bad in [(-1, 1, 64), (1, 0, 64), (1, 65, 64), (1, 1, -1)]:
        assert B.ct_packed_attention_workspace_bytes(c, *bad) == 0


# ---------------------------------------------------------------------------------- refusals
def test_pack_refusals():
    c = _cfg()

    def call(k=FAKE, ks=1024, v=FAKE, vs=1024, n=8, rows=FAKE, first=0, cache=FAKE, n_rows=64, bits=4):
        return _status(B.ct_pack_kv, c, k, ks, v, vs, n, rows, first, cache, n_rows, bits)

    assert call(n=-1) == B.CT_ERR_SHAPE
    assert call(bits=2) == B.CT_ERR_UNSUPPORTED
    assert call(n_rows=40) == B.CT_ERR_SHAPE and call(n_rows=0) == B.CT_ERR_SHAPE
    assert call(k=None) == B.CT_ERR_NULL and call(v=None) == B.CT_ERR_NULL and call(cache=None) == B.CT_ERR_NULL
    assert call(ks=1023) == B.CT_ERR_SHAPE and call(vs=0) == B.CT_ERR_SHAPE
    assert call(ks=1028) == B.CT_ERR_UNSUPPORTED
    assert call(k=FAKE + 8) == B.CT_ERR_UNSUPPORTED and call(cache=FAKE + 4) == B.CT_ERR_UNSUPPORTED
    assert call(rows=None, first=57) == B.CT_ERR_INDEX and call(rows=None, first=-1) == B.CT_ERR_INDEX
    assert call(rows=None, first=0x7fffffff) == B.CT_ERR_INDEX
    assert _status(B.ct_pack_kv, _cfg(head_dim=96), FAKE, 1024, FAKE, 1024, 8, FAKE, 0, FAKE, 64, 4) == B.CT_ERR_UNSUPPORTED
    B.ct_pack_kv(c, None, 1024, None, 1024, 0, None, 0, None, 64, 4)            # empty work is legal and needs no GPU


def test_unpack_refusals():
    c = _cfg()

    def call(cache=FAKE, n_rows=64, bits=8, rows=FAKE, first=0, old=FAKE, new=FAKE, n=8, k=FAKE, v=FAKE):
        return _status(B.ct_unpack_kv, c, cache, n_rows, bits, rows, first, old, new, n, k, v)

    assert call(n=-1) == B.CT_ERR_SHAPE and call(n_rows=63) == B.CT_ERR_SHAPE and call(bits=0) == B.CT_ERR_UNSUPPORTED
    assert call(cache=None) == B.CT_ERR_NULL and call(k=None) == B.CT_ERR_NULL and call(v=None) == B.CT_ERR_NULL
    assert call(new=None) == B.CT_ERR_NULL                                      # old positions without new ones
    assert call(rows=None, first=60) == B.CT_ERR_INDEX
    assert call(k=FAKE + 2) == B.CT_ERR_UNSUPPORTED
    B.ct_unpack_kv(c, None, 64, 4, None, 0, None, None, 0, None, None)


def test_attention_refusals():
    c = _cfg()

    def call(cfg=c, q=FAKE, n_seq=2, n_new=1, cache=FAKE, n_rows=65536, bits=4, start=FAKE, length=FAKE, max_len=32768, out=FAKE,
             ws=None, ws_bytes=0):
        return _status(B.ct_packed_attention, cfg, q, n_seq, n_new, cache, n_rows, bits, start, length, max_len, out, None, ws, ws_bytes)

    need = B.ct_packed_attention_workspace_bytes(c, 2, 1, 32768)
    assert need > 0
    assert call() == B.CT_ERR_WORKSPACE
    assert call(ws=FAKE, ws_bytes=need - 1) == B.CT_ERR_WORKSPACE
    assert call(ws=FAKE + 64, ws_bytes=need) == B.CT_ERR_WORKSPACE
    assert call(n_seq=-1) == B.CT_ERR_SHAPE and call(max_len=-1) == B.CT_ERR_SHAPE and call(n_new=0) == B.CT_ERR_SHAPE
    assert call(n_new=65) == B.CT_ERR_UNSUPPORTED
    assert call(n_seq=1 << 26) == B.CT_ERR_UNSUPPORTED                          # rows beyond one launch
    assert call(max_len=65537) == B.CT_ERR_SHAPE
    assert call(bits=3) == B.CT_ERR_UNSUPPORTED and call(n_rows=100) == B.CT_ERR_SHAPE
    for name in ("q", "cache", "start", "length", "out"):
        assert call(**{name: None}) == B.CT_ERR_NULL
    assert call(q=FAKE + 8) == B.CT_ERR_UNSUPPORTED
    assert call(cfg=_cfg(n_q_heads=24)) == B.CT_ERR_UNSUPPORTED
    B.ct_packed_attention(c, None, 0, 1, None, 64, 4, None, None, 64, None, None, None, 0)


def test_launches_beyond_what_a_grid_holds_are_refused():
    """A launch has fewer than 2^32 threads."""
    c, most = _cfg(), 2 ** 31 - 1
    assert _status(B.ct_pack_kv, c, FAKE, 1024, FAKE, 1024, most, FAKE, 0, FAKE, 64, 4) == B.CT_ERR_UNSUPPORTED
    assert _status(B.ct_unpack_kv, c, FAKE, 64, 4, FAKE, 0, None, None, most, FAKE, FAKE) == B.CT_ERR_UNSUPPORTED
    assert _status(B.ct_qk_norm_rope, c, FAKE, FAKE, most, FAKE, FAKE, 0.0, FAKE, FAKE, FAKE) == B.CT_ERR_UNSUPPORTED
    rows = 2 ** 32 // 256 // 32                                                 # sequences whose rows just do not fit
    assert _status(B.ct_packed_attention, c, FAKE, rows, 1, FAKE, 64, 4, FAKE, FAKE, 64, FAKE, None, None, 0) == B.CT_ERR_UNSUPPORTED
    assert _status(B.ct_packed_attention, c, FAKE, rows - 1, 1, FAKE, 64, 4, FAKE, FAKE, 64, None, None, None, 0) == B.CT_ERR_NULL


def test_qk_norm_refusals():
    c = _cfg()

    def call(qkv=FAKE, pos=FAKE, n=4, qw=FAKE, kw=FAKE, eps=1e-6, q=FAKE, k=FAKE, v=FAKE):
        return _status(B.ct_qk_norm_rope, c, qkv, pos, n, qw, kw, eps, q, k, v)

    assert call(n=-1) == B.CT_ERR_SHAPE
    assert call(eps=-1.0) == B.CT_ERR_SHAPE and call(eps=float("nan")) == B.CT_ERR_SHAPE and call(eps=float("inf")) == B.CT_ERR_SHAPE
    for name in ("qkv", "pos", "qw", "kw", "q", "k"):
        assert call(**{name: None}) == B.CT_ERR_NULL
    for name in ("qkv", "qw", "kw", "q", "k", "v"):
        assert call(**{name: FAKE + 2}) == B.CT_ERR_UNSUPPORTED
    B.ct_qk_norm_rope(c, None, None, 0, None, None, 1e-6, None, None, None)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128), (16, 1, 128), (16, 16, 64), (2, 1, 64), (64, 8, 128)])
def test_one_workspace_is_enough_for_attention_of_every_size(hq, hkv, d):
    cfg = B.make_cfg(hq * d, hq, hkv, d, 1e4, 0, 0.0)
    for n_new in (1, 2, 4, 5, 8, 9, 17, 33, 64):
        for n_seq in [*range(1, 66), 100, 128, 200, 255, 256, 257, 300, 1000]:
            for max_len in (0, 1, 1024, 1025, 2049, 4099, 8192, 8225, 65536, 1 << 20, 1 << 30):
                need = B.ct_packed_attention_workspace_bytes(cfg, n_seq, n_new, max_len)
                assert 0 <= need <= 65536 * (d + 2), (n_seq, n_new, max_len, need)
