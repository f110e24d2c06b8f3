"""Calls over packed caches ordered on a stream of their own: everything that they read is made there just before, and
what they write is used there right after, so a call on any other stream would meet wrong inputs."""
import numpy as np
import pytest
import torch

from oracle import ct_oracle as O
from paper_2605_24022_amd import binding as B
from paper_2605_24022_amd import workloads as W
from tests.gpu_util import dev_bf16, dev_i32, f64_of, say
from tests.test_gpu_packed import _bits, _held_to_oracle, _rope_bound, _same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    assert torch.cuda.is_available()
    B.load()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("top", [400, 3000])      # the key range whole, and in parts
def test_inputs_made_and_outputs_used_on_a_side_stream(top):
    """Context rows and a decoding step: pack, read back and rotate, project's rows normed, the new row appended, attention."""
    hq, hkv, d, bits, n, n_rows = 32, 8, 128, 8, 300, 3008
    say(f"packed calls ordered on a side stream, max_len={top}")
    rng = np.random.default_rng(top)
    cfg = B.make_cfg(hq * d, hq, hkv, d, 1e4, 0, 0.0)
    o = (hq + 2 * hkv) * d
    need = B.ct_packed_attention_workspace_bytes(cfg, 1, 1, top)
    assert (need > 0) == (top > 1024)
    host = {"k": _bits(rng, n, hkv, d), "v": _bits(rng, n, hkv, d), "qkv": _bits(rng, 1, o),
            "w": W.f32_to_bf16_bits((1 + 0.3 * rng.standard_normal(d)).astype(np.float32))}
    ints = {"start": [0], "length": [n + 1], "new": rng.integers(0, 100000, n), "pos": [n], "row": [n]}
    right = {**{x: dev_bf16(a) for x, a in host.items()}, **{x: dev_i32(a) for x, a in ints.items()}}
    read = {x: torch.zeros_like(t) for x, t in right.items()}       # what the calls read: zeros until the stream fills them
    bf16 = {"dtype": torch.bfloat16, "device": "cuda"}
    wrote = {"k2": torch.zeros((n, hkv, d), **bf16), "v2": torch.zeros((n, hkv, d), **bf16), "q": torch.zeros((1, 1, hq, d), **bf16),
             "k1": torch.zeros((1, hkv, d), **bf16), "out": torch.zeros((1, 1, hq, d), **bf16)}
    used = {x: torch.zeros_like(t) for x, t in wrote.items()}
    cache = torch.full((B.ct_packed_kv_bytes(cfg, n_rows, bits),), 0xff, dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    big = torch.zeros(1 << 28, device="cuda")
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for _ in range(16):
            big += 1                                                 # some milliseconds ahead of everything
        for x, t in read.items():
            t.copy_(right[x])
        B.ct_pack_kv(cfg, read["k"], hkv * d, read["v"], hkv * d, n, None, 0, cache, n_rows, bits, st)
        B.ct_unpack_kv(cfg, cache, n_rows, bits, None, 0, None, read["new"], n, wrote["k2"], wrote["v2"], st)
        B.ct_qk_norm_rope(cfg, read["qkv"], read["pos"], 1, read["w"], read["w"], 1e-6, wrote["q"], wrote["k1"], None, st)
        B.ct_pack_kv(cfg, wrote["k1"], hkv * d, read["qkv"][:, (hq + hkv) * d:], o, 1, read["row"], 0, cache, n_rows, bits, st)
        B.ct_packed_attention(cfg, wrote["q"], 1, 1, cache, n_rows, bits, read["start"], read["length"], top, wrote["out"], None, ws, need, st)
        for x, t in used.items():
            t.copy_(wrote[x])
    st.synchronize()
    got = {x: f64_of(t) for x, t in used.items()}
    kv, vv = (O.packed_values(W.bf16_bits_to_f64(host[x]), bits) for x in ("k", "v"))
    _same(got["v2"], vv, "V read back")
    turned = O.rotate(kv, ints["new"], 1e4, 0)
    assert (np.abs(got["k2"] - turned) <= _rope_bound(turned, d, 0)).all(), "K read back"
    wf = W.bf16_bits_to_f64(host["w"])
    wq, wk, wv = O.qk_norm_rope(W.bf16_bits_to_f64(host["qkv"]), [n], wf, wf, 1e-6, hq, hkv, d, 1e4)
    for x, want in (("q", wq[None]), ("k1", wk)):
        assert (np.abs(got[x] - want) <= _rope_bound(want, d, 0) + 2.0 ** -18 * np.abs(want)).all(), x
    keys = np.concatenate([kv, O.packed_values(got["k1"], bits)])
    values = np.concatenate([vv, O.packed_values(wv, bits)])
    _held_to_oracle(got["out"][0], got["q"][0], keys, values, "attention")
