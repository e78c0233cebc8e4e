"""Sizes of the attention over the cache, on the host: products that pass 64 bits, workspaces of growing sequences."""
import ctypes as C

import pytest

from paper_2411_17686_amd import ficoco as fc
from tests.test_cache_abi import _attention, _bytes, _cache


@pytest.mark.parametrize("B,H,heads,n_q", [(1 << 30, 1 << 15, 1 << 15, 1 << 26), ((1 << 31) - 1, 65535, 65535, 1 << 29), (1 << 16, 4, 4, 1 << 13), (1, 4, 4, 1 << 29)])
def test_too_many_rows_are_refused(B, H, heads, n_q):
    """(the first would be 2^64 workgroups, zero in 64 bits, by which a plan must not divide)"""
    a = _attention(B=B, H=H, n_q=n_q, Q=1 << 60, O=1 << 55, q_stride_b=0, q_stride_h=0, q_stride_n=0, o_stride_b=1 << 52, o_stride_h=1 << 36, o_stride_n=128)
    assert _bytes(fc.lib().ficoco_cache_attention_workspace_bytes, C.byref(_cache(heads=heads)), C.byref(a))[0] == fc.EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(), dict(B=1), dict(n_q=3), dict(n_q=30), dict(n_q=200, o_stride_h=200 * 128, o_stride_b=8 * 200 * 128), dict(window=3000), dict(window=500, sinks=4, n_q=8)])
def test_a_workspace_serves_every_shorter_sequence(kw):
    """max_len grows with the sequences of a decoder; 0 stands for the longest."""
    kw = dict(kw, O=1 << 40)
    size = lambda n: _bytes(fc.lib().ficoco_cache_attention_workspace_bytes, C.byref(_cache(max_pages=2000)), C.byref(_attention(max_len=n, **kw)))
    sizes = [size(n) for n in list(range(1, 4000, 37)) + [10000, 50000, 128000, 1 << 30, 0]]
    assert all(rc == fc.OK for rc, _ in sizes)
    assert [b for _, b in sizes] == sorted(b for _, b in sizes)
