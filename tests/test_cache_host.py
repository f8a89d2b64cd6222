"""What the calls of include/catekv_cache.h refuse, on the host: arguments are
checked before the GPU is touched.  The 64-bit forms that the GPU tests compare
with are pinned here by facts other than their own formulas."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2608_30295_amd as ck
from paper_2608_30295_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "catekv_cache.h")
needs_lib = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libcatekv.so not built")

FAKE = 0x100000   # a non-null pointer value; never dereferenced on these paths
INVALID, UNSUPPORTED, WORKSPACE = _lib.CATEKV_ERR_INVALID_ARG, _lib.CATEKV_ERR_UNSUPPORTED, _lib.CATEKV_ERR_WORKSPACE


def plan_of(batch=1, hq=8, hkv=2, ws_bytes=1 << 12):
    p = _lib.DecodePlanT()
    p.magic = 0x43617465504c414e                    # a plan header as catekv_decode_plan fills it
    p.batch, p.hq, p.hkv, p.ws_bytes, p.n_workers, p.variant = batch, hq, hkv, ws_bytes, 4, 2
    p.max_len_total = 1000
    return p


@needs_lib
def test_every_declared_symbol_is_exported_with_its_signature():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(catekv_[a-z_0-9]+)\s*\(", text)))
    assert set(names) == set(_lib.CACHE_SIGNATURES) and len(names) == 9
    for n in names:
        args = re.search(n + r"\s*\(([^)]*)\)", text, flags=re.S).group(1)
        assert len(args.split(",")) == len(_lib.CACHE_SIGNATURES[n][1]), n
        assert hasattr(ck.lib(), n)


CONVERT = dict(format=0, dtype=1, block=64, kv=FAKE, lens=FAKE, views=FAKE, n_views=2, max_rows=100, d=128)


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(format=2), UNSUPPORTED), (dict(format=-1), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(block=16), INVALID), (dict(block=128), INVALID), (dict(block=0), INVALID),
    (dict(kv=None), INVALID), (dict(lens=None), INVALID), (dict(views=None), INVALID),
    (dict(n_views=0), INVALID), (dict(n_views=-3), INVALID), (dict(max_rows=0), INVALID),
    (dict(max_rows=1 << 31), UNSUPPORTED), (dict(d=64), UNSUPPORTED),
    (dict(n_views=1 << 20, max_rows=1 << 30), UNSUPPORTED),
])
def test_conversions_refuse(change, status):
    a = {**CONVERT, **change}
    L = ck.lib()
    assert L.catekv_q8_quantize(a["format"], a["dtype"], a["block"], a["kv"], a["lens"], a["views"], a["n_views"],
                                a["max_rows"], a["d"], None) == status
    assert L.catekv_last_error()
    assert L.catekv_q8_dequantize(a["format"], a["dtype"], a["block"], a["views"], a["lens"], a["kv"], a["n_views"],
                                  a["max_rows"], a["d"], None) == status


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(format=7), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(block=8), INVALID),
    (dict(views=None), INVALID), (dict(capacity=None), INVALID), (dict(lens=None), INVALID), (dict(k=None), INVALID),
    (dict(v=None), INVALID), (dict(batch=0), INVALID), (dict(hkv=0), INVALID), (dict(d=256), UNSUPPORTED),
    (dict(batch=1 << 20, hkv=1 << 20), INVALID), (dict(k=FAKE + 8), INVALID), (dict(v=FAKE + 2), INVALID),
])
def test_append_refuses(change, status):
    a = dict(format=1, dtype=0, block=32, views=FAKE, capacity=FAKE, lens=FAKE, k=FAKE, v=FAKE, batch=1, hkv=2, d=128)
    a.update(change)
    assert ck.lib().catekv_q8_append(a["format"], a["dtype"], a["block"], a["views"], a["capacity"], a["lens"], a["k"],
                                     a["v"], a["batch"], a["hkv"], a["d"], None, None) == status


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(plan=_lib.DecodePlanT()), INVALID), (dict(q=None), INVALID), (dict(views=None), INVALID),
    (dict(lens=None), INVALID), (dict(out=None), INVALID), (dict(batch=2), INVALID), (dict(hq=16), INVALID),
    (dict(hq=6), UNSUPPORTED), (dict(d=64), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(decay=-0.1), INVALID), (dict(decay=1.5), INVALID),
    (dict(decay=float("nan")), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 8), WORKSPACE),
    (dict(ws_bytes=100), WORKSPACE), (dict(wws=None), WORKSPACE), (dict(wws=FAKE + 64), WORKSPACE),
    (dict(wws_bytes=64), WORKSPACE), (dict(q=FAKE + 8), INVALID), (dict(out=FAKE + 4), INVALID),
])
def test_attention_refuses(change, status):
    a = dict(dtype=1, plan=plan_of(), q=FAKE, views=FAKE, lens=FAKE, batch=1, hq=8, hkv=2, d=128, scale=0.1, out=FAKE,
             acc=FAKE, decay=1.0, ws=FAKE, ws_bytes=1 << 20, wws=FAKE, wws_bytes=1 << 20)
    a.update(change)
    L = ck.lib()
    rest = (ctypes.byref(a["plan"]), a["q"], a["views"], a["lens"], a["batch"], a["hq"], a["hkv"], a["d"], a["scale"],
            a["out"], None, a["acc"], a["decay"], a["ws"], a["ws_bytes"], a["wws"], a["wws_bytes"], None)
    assert L.catekv_decode_attn_weights(a["dtype"], *rest) == status
    assert L.catekv_q8_decode_attn(0, a["dtype"], 64, *rest) == status
    assert L.catekv_last_error()


@needs_lib
def test_attention_refuses_what_each_call_has_of_its_own():
    L, p = ck.lib(), plan_of()
    rest = (ctypes.byref(p), FAKE, FAKE, FAKE, 1, 8, 2, 128, 0.1, FAKE, None)
    end = (1.0, FAKE, 1 << 20, FAKE, 1 << 20, None)
    assert L.catekv_decode_attn_weights(1, *rest, None, *end) == INVALID        # no weights asked for
    assert L.catekv_q8_decode_attn(2, 1, 64, *rest, FAKE, *end) == UNSUPPORTED
    assert L.catekv_q8_decode_attn(0, 1, 48, *rest, FAKE, *end) == INVALID
    assert L.catekv_weights_workspace(ctypes.byref(_lib.DecodePlanT())) == 0
    # rows of a share: at most ceil((1000 + 2 63) / 64) units over 4 workers, 4 heads, fp32
    assert L.catekv_weights_workspace(ctypes.byref(p)) == 5 * 64 * 4 * 4 * 4


EVICT = dict(views=FAKE, lens=FAKE, acc=FAKE, budget=FAKE, n=2, max_rows=1000, cs=64, recent=0, d=128, ws=FAKE, wsb=1 << 20)


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(views=None), INVALID), (dict(lens=None), INVALID), (dict(acc=None), INVALID), (dict(budget=None), INVALID),
    (dict(n=0), INVALID), (dict(n=1 << 17), UNSUPPORTED), (dict(max_rows=0), INVALID), (dict(max_rows=-5), INVALID),
    (dict(max_rows=1 << 27), UNSUPPORTED), (dict(max_rows=1 << 40), UNSUPPORTED), (dict(cs=0), INVALID),
    (dict(cs=-8), INVALID), (dict(cs=1 << 21), UNSUPPORTED), (dict(recent=-1), INVALID), (dict(d=127), UNSUPPORTED),
    (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 16), WORKSPACE), (dict(wsb=10), WORKSPACE),
])
def test_evict_refuses(change, status):
    a = {**EVICT, **change}
    rest = (a["views"], a["lens"], a["acc"], a["budget"], a["n"], a["max_rows"], a["cs"], a["recent"], a["d"], a["ws"],
            a["wsb"], None)
    assert ck.lib().catekv_evict_kv(1, *rest) == status
    assert ck.lib().catekv_q8_evict(64, *rest) == status
    assert ck.lib().catekv_last_error()


@needs_lib
def test_evict_refuses_what_each_call_has_of_its_own():
    L = ck.lib()
    rest = lambda cs: (FAKE, FAKE, FAKE, FAKE, 2, 1000, cs, 0, 128, FAKE, 1 << 20, None)
    assert L.catekv_evict_kv(5, *rest(8)) == UNSUPPORTED
    assert L.catekv_q8_evict(16, *rest(64)) == INVALID
    assert L.catekv_q8_evict(64, *rest(32)) == INVALID                          # half a block
    assert L.catekv_q8_evict(32, *rest(40)) == INVALID
    assert ck.evict_workspace(0, 100, 8) == ck.evict_workspace(2, 0, 8) == ck.evict_workspace(2, 100, 0) == 0
    assert ck.evict_workspace(2, 1 << 27, 8) == 0 and ck.evict_workspace(2, 100, 8) > 0


@needs_lib
def test_the_binding_refuses_before_the_library():
    i64, f32 = torch.int64, torch.float32
    for kw in (dict(fmt="int4"), dict(block=16), dict(dtype=torch.float16)):
        with pytest.raises((ValueError, TypeError)):
            ck.q8_views([[1] * 6], "cpu", **{**dict(fmt="int8", block=32, dtype=f32), **kw})
    with pytest.raises(ValueError):
        ck.q8_views([[1] * 5], "cpu", fmt="int8", block=32, dtype=f32)
    with pytest.raises(ValueError):
        ck.q8_views([], "cpu", fmt="int8", block=32, dtype=f32)
    q8 = ck.q8_views([[1] * 6] * 2, "cpu", fmt="int8", block=32, dtype=f32)
    host = torch.zeros(2, dtype=i64)
    for call in (lambda: ck.quantize_kv(torch.zeros((2, 2), dtype=i64), host, q8, 10),
                 lambda: ck.dequantize_kv(q8, host, torch.zeros((2, 2), dtype=i64), 10),
                 lambda: ck.append_kv_q8(q8, host, host, torch.zeros(1, 2, 128), torch.zeros(1, 2, 128)),
                 lambda: ck.evict_kv(torch.zeros((2, 2), dtype=i64), host, host, host, cs=8, recent=0, max_rows=10,
                                     dtype=f32),
                 lambda: ck.evict_kv_q8(q8, host, host, host, cs=32, recent=0, max_rows=10)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError):
        ck.evict_kv(torch.zeros((2, 2), dtype=i64), host, host, host, cs=8, recent=0, max_rows=10, dtype=torch.float16)


# ----------------------------------------------------------- the 64-bit forms themselves

def test_e4m3_values_are_torch_s():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(R.e4m3_value(codes).astype(np.float32), want, equal_nan=True)


def test_e4m3_codes_are_torch_s_conversion():
    # with a power-of-two scale the quotient is exact, so that a library conversion is the same rounding
    x = np.random.default_rng(1).standard_normal((64, 128)) * np.exp(np.random.default_rng(2).uniform(-9, 3, (64, 128)))
    x = x.astype(np.float32)
    s = R.block_scale(x.astype(np.float64), "e4m3")
    assert np.log2(s) == int(np.log2(s)) and 224 * s < np.abs(x).max() <= 448 * s
    want = torch.from_numpy(x / s).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.block_codes(x.astype(np.float64), "e4m3", s), want)


def test_int8_codes_by_hand():
    x = np.zeros((32, 128))
    x[0, :6] = [127, 0.5, 1.5, -2.5, -0.5, 63.49]
    s = R.block_scale(x, "int8")
    assert s == np.float32(127) * np.float32(1 / 127)      # one or one bit beside it
    codes = R.block_codes(x, "int8", np.float32(1)).view(np.int8)
    assert codes[0, :6].tolist() == [127, 0, 2, -2, 0, 63]   # ties to even
    assert R.block_scale(np.zeros((32, 128)), "int8") == 0
    assert np.isnan(R.block_scale(np.full((32, 128), np.inf), "e4m3"))


def test_eviction_by_hand():
    # chunks of 2: weights 5, 9, 1, 4, 8 and one row behind; three stay: 9 (1), 8 (4), 5 (0)
    acc = [5, 0, 0, 9, 1, 1, 4, 0, 8, 2, 7]
    assert R.evict(np.array(acc, dtype=float), 3, 2, 1).tolist() == [0, 1, 2, 3, 8, 9, 10]
    assert R.evict(np.array(acc, dtype=float), 1, 2, 1).tolist() == [2, 3, 10]          # 9 takes place 0
    assert R.evict(np.array(acc, dtype=float), 0, 2, 1).tolist() == [10]
    assert R.evict(np.array(acc, dtype=float), 5, 2, 1).tolist() == list(range(11))
    assert R.evict(np.array(acc, dtype=float), 2, 2, 7).tolist() == list(range(11))     # two compete, two stay
    assert R.evict(np.array([1.0, 1, 1, 1]), 2, 1, 0).tolist() == [0, 1]                # ties: the lower one
    assert R.evict(np.array([1.0, np.nan, np.inf, 3]), 2, 1, 0).tolist() == [2, 1]      # NaN above inf


def test_attention_form_against_a_library():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, 128, generator=g, dtype=torch.float64) for n in (4, 50, 50))
    out, lse, w, _, _ = R.attend(q.numpy(), k.numpy(), v.numpy(), 0.125)
    ref = torch.nn.functional.scaled_dot_product_attention(q[None], k[None], v[None], scale=0.125)[0]
    assert np.allclose(out, ref.numpy(), rtol=0, atol=1e-12) and abs(w.sum() - 1) < 1e-12
    assert np.allclose(lse, torch.logsumexp(q @ k.T * 0.125, dim=1).numpy(), atol=1e-12)
