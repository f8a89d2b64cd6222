"""Sizes at which the calls of include/catekv_cache.h would need a launch of 2^32
threads or more, which HIP does not take: refused on the host, before any launch."""
import ctypes
import os

import numpy as np
import pytest

import paper_2608_30295_amd as ck
from paper_2608_30295_amd import _lib

pytestmark = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libcatekv.so not built")

FAKE = 0x100000   # a non-null pointer value; never dereferenced on these paths
INVALID, UNSUPPORTED = _lib.CATEKV_ERR_INVALID_ARG, _lib.CATEKV_ERR_UNSUPPORTED
HUGE = 1 << 60


@pytest.mark.parametrize("n_views,max_rows,cs", [
    (16384, 1 << 20, 64),             # keys: 256 workgroups of 1024 threads per view
    (65536, 1 << 26, 64), (65536, 1 << 20, 4096), (65536, 1 << 26, 1 << 20),
    (16384, 1 << 20, 1), (8192, 1 << 21, 8),
    (8192, 1 << 24, 1 << 20),         # keys fit, the zeros behind the new lengths do not
    (6000, 1 << 21, 2112),            # one chunk per workgroup of the keys: twice as many as of 4096 rows
])
def test_evictions_that_no_launch_takes(n_views, max_rows, cs):
    L = ck.lib()
    assert ck.evict_workspace(n_views, max_rows, cs) == 0
    rest = (FAKE, FAKE, FAKE, FAKE, n_views, max_rows, cs, 0, 128, FAKE, HUGE, None)
    assert L.catekv_evict_kv(1, *rest) == UNSUPPORTED
    assert L.catekv_q8_evict(64, *rest) == UNSUPPORTED


def test_evictions_just_below_the_limit_have_a_workspace():
    for n_views, max_rows, cs in ((16383, 1 << 20, 64), (8191, 1 << 21, 8), (4095, 1 << 22, 1), (65536, 1 << 16, 8),
                                  (65536, 16384, 1), (64, 1 << 26, 64)):
        assert ck.evict_workspace(n_views, max_rows, cs) > 0, (n_views, max_rows, cs)
    # as the header states: whatever cs is, while n_views * max_rows is at most 2^32
    for cs in (1, 7, 64, 2049, 4096, 4097, 100_000, 1 << 20):
        for n_views in (64, 4096, 65536):
            assert ck.evict_workspace(n_views, (1 << 32) // n_views, cs) > 0, (n_views, cs)


@pytest.mark.parametrize("block,n_views,max_rows", [
    (64, 4096, 1 << 20),              # 4097 workgroups of 256 threads per view: 4095 views are the most
    (32, 2048, 1 << 20), (32, 16, (1 << 31) - 1), (64, 1 << 24, 1), (64, 1 << 22, 1000),
])
def test_conversions_that_no_launch_takes(block, n_views, max_rows):
    L = ck.lib()
    assert L.catekv_q8_quantize(0, 1, block, FAKE, FAKE, FAKE, n_views, max_rows, 128, None) == UNSUPPORTED
    assert L.catekv_q8_dequantize(1, 0, block, FAKE, FAKE, FAKE, n_views, max_rows, 128, None) == UNSUPPORTED


def test_appends_that_no_launch_takes():
    # 512 threads per view
    for batch, hkv in ((1 << 20, 8), (1 << 23, 1), (1 << 24, 127)):
        assert ck.lib().catekv_q8_append(1, 0, 32, FAKE, FAKE, FAKE, FAKE, FAKE, batch, hkv, 128, None, None) == INVALID
        assert "too large" in ck.lib().catekv_last_error().decode()


def plan_of(batch, hq, hkv, n_workers, n_multi):
    p = _lib.DecodePlanT()
    p.magic = 0x43617465504c414e                    # a plan header as catekv_decode_plan fills it
    p.batch, p.hq, p.hkv, p.ws_bytes, p.n_workers, p.n_multi, p.variant = batch, hq, hkv, 1 << 12, n_workers, n_multi, 1
    p.max_len_total = 1000
    return p


@pytest.mark.parametrize("batch,hq,hkv,n_workers,n_multi", [
    (1, 8, 2, 1 << 23, 0),            # the stream: 512 threads per worker
    (1 << 20, 8, 8, 4, 1),            # the join: as many per view and head, where a view has several parts
    (1 << 18, 32, 4, 4, 1), (1 << 16, 8, 2, (1 << 23) - (1 << 19), 1),
])
def test_attention_steps_that_no_launch_takes(batch, hq, hkv, n_workers, n_multi):
    L, p = ck.lib(), plan_of(batch, hq, hkv, n_workers, n_multi)
    rest = (ctypes.byref(p), FAKE, FAKE, FAKE, batch, hq, hkv, 128, 0.1, FAKE, None, FAKE, 1.0, FAKE, HUGE, FAKE, HUGE, None)
    assert L.catekv_decode_attn_weights(1, *rest) == UNSUPPORTED
    assert L.catekv_q8_decode_attn(0, 1, 64, *rest) == UNSUPPORTED


def test_partials_lie_on_16_byte_borders():
    """The kernels that join a view's partials read them 16 bytes at a time.  A plan's bytes
    differ between group sizes by its partials alone: 256 parts, each o [G][128], m [G] and
    l [G] in fp32."""
    def total(G):
        n = np.array([256 * 64], dtype=np.int64)
        return ck.lib().catekv_decode_workspace(n.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), 1, G, 1, 64)
    more = [(total(G) - total(8)) / 256 for G in (1, 2, 4)]
    eight = 4 * (8 * 128 + 2 * 8)
    assert eight % 16 == 0
    for G, m in zip((1, 2, 4), more):
        assert (eight + m) % 16 == 0 and 0 <= eight + m - 4 * (G * 128 + 2 * G) < 16, G
