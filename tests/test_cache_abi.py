"""The cache's part of the ABI without a GPU: layouts of its structs, sizes of workspaces, and what is refused on the host."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2411_17686_amd import ficoco as fc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name,mirror", [("ficoco_cache", fc.CacheProblem), ("ficoco_tokens", fc.TokensProblem),
                                         ("ficoco_attention", fc.AttentionProblem)])
def test_struct_layouts_match_the_header(tmp_path, name, mirror):
    fields = [f[0] for f in mirror._fields_]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ficoco.h"', "int main(void){",
             'printf("%%zu\\n", sizeof(%s));' % name]
    lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f in fields] + ["return 0;}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert out[0] == C.sizeof(mirror)
    assert out[1:] == [getattr(mirror, f).offset for f in fields]
    packed = {"ficoco_tokens": fc._TOKENS, "ficoco_attention": fc._ATTENTION}.get(name)       # (what the binding passes)
    if packed is not None:
        values = [float(3 * i + 1) if t is C.c_float else 3 * i + 1 for i, (_, t) in enumerate(mirror._fields_)]
        assert packed.size == out[0] and packed.pack(*values) == bytes(mirror(*values))


def _cache(**kw):
    c = fc.CacheProblem(2, 100, 64, 4, 128, 10, 20, 4096, 8192, 16, 32, 64, 128, 256)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _attention(**kw):
    a = fc.AttentionProblem(B=3, H=8, H_kv=4, n_q=1, n_k=50, d_head=128, Q=4096, K=1 << 20, V=1 << 21, O=1 << 30, scale=0.1)
    for p in "qkvo":
        setattr(a, p + "_stride_b", 8 * 50 * 128)
        setattr(a, p + "_stride_h", 50 * 128)
        setattr(a, p + "_stride_n", 128)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _bytes(fn, *args):
    n = C.c_size_t()
    return fn(*args, C.byref(n)), n.value


@pytest.mark.parametrize("code,kw", [
    (fc.EINVAL, dict(layers=0)), (fc.EINVAL, dict(n_pages=0)), (fc.EINVAL, dict(heads=-1)), (fc.EINVAL, dict(n_seqs=0)),
    (fc.EINVAL, dict(max_pages=0)), (fc.EINVAL, dict(k=None)), (fc.EINVAL, dict(v=4104)), (fc.EINVAL, dict(k_exp=None)),
    (fc.EINVAL, dict(table=None)), (fc.EINVAL, dict(refs=258)), (fc.EINVAL, dict(len=None)),
    (fc.EUNSUPPORTED, dict(page_size=8)), (fc.EUNSUPPORTED, dict(page_size=48)), (fc.EUNSUPPORTED, dict(page_size=256)),
    (fc.EUNSUPPORTED, dict(d_head=96)), (fc.EUNSUPPORTED, dict(d_head=32)), (fc.EUNSUPPORTED, dict(n_seqs=8193)),
    (fc.EUNSUPPORTED, dict(max_pages=1 << 26))])
def test_cache_refusals(code, kw):
    L = fc.lib()
    assert _bytes(L.ficoco_cache_workspace_bytes, C.byref(_cache(**kw)), 3)[0] == code
    assert _bytes(L.ficoco_cache_attention_workspace_bytes, C.byref(_cache(**kw)), C.byref(_attention()))[0] == code


def test_workspace_sizes():
    L = fc.lib()
    rc, n = _bytes(L.ficoco_cache_workspace_bytes, C.byref(_cache()), 3)
    assert rc == fc.OK and n >= 3 * 20 * 4
    assert _bytes(L.ficoco_cache_workspace_bytes, C.byref(_cache()), 1025)[0] == fc.EINVAL
    assert _bytes(L.ficoco_cache_workspace_bytes, C.byref(_cache()), -1)[0] == fc.EINVAL
    size = lambda **kw: _bytes(L.ficoco_cache_attention_workspace_bytes, C.byref(_cache(max_pages=2000)), C.byref(_attention(**kw)))
    short, long = size(max_len=200), size(max_len=100000)
    assert short[0] == long[0] == fc.OK and 0 < short[1] < long[1]
    assert size(max_len=100000, window=100)[1] == short[1]
    assert size(B=0) == (fc.OK, size(B=0)[1])


@pytest.mark.parametrize("code,kw", [
    (fc.EINVAL, dict(B=-1)), (fc.EINVAL, dict(n_q=-1)), (fc.EINVAL, dict(H=0)), (fc.EINVAL, dict(H=6)), (fc.EINVAL, dict(d_head=64)),
    (fc.EINVAL, dict(window=-1)), (fc.EINVAL, dict(sinks=-1)), (fc.EINVAL, dict(max_len=-1)), (fc.EINVAL, dict(scale=0.0)),
    (fc.EINVAL, dict(scale=-1.0)), (fc.EINVAL, dict(scale=float("nan"))), (fc.EINVAL, dict(scale=float("inf"))),
    (fc.EINVAL, dict(q_stride_h=-128)), (fc.EINVAL, dict(o_stride_h=64)), (fc.EINVAL, dict(o_stride_b=0)), (fc.EINVAL, dict(Q=None)),
    (fc.EINVAL, dict(O=None)), (fc.EINVAL, dict(Q=4097)), (fc.EINVAL, dict(O=4096)), (fc.EINVAL, dict(n_q=2, o_stride_n=100)),
    (fc.EINVAL, dict(n_q=1 << 30)), (fc.EUNSUPPORTED, dict(n_q=1 << 30, O=1 << 50))])
def test_attention_refusals(code, kw):
    assert _bytes(fc.lib().ficoco_cache_attention_workspace_bytes, C.byref(_cache()), C.byref(_attention(**kw)))[0] == code


def test_null_contexts_are_refused():
    L = fc.lib()
    assert L.ficoco_cache_reserve(None, C.byref(_cache()), 1, None, None, 1, None, None) == fc.EINVAL
    assert L.ficoco_cache_append(None, C.byref(_cache()), 0, None, None) == fc.EINVAL
    assert L.ficoco_cache_read(None, C.byref(_cache()), 0, None, None) == fc.EINVAL
    assert L.ficoco_cache_fork(None, C.byref(_cache()), 1, None, None, 0, None, None) == fc.EINVAL
    assert L.ficoco_cache_compact(None, C.byref(_cache()), 0, 1, 1, None, None, 0, 1, 1, None, None, None, 0, None) == fc.EINVAL
    assert L.ficoco_cache_free(None, C.byref(_cache()), 1, None, None) == fc.EINVAL
    assert L.ficoco_cache_attention(None, C.byref(_cache()), 0, C.byref(_attention()), None, 0, None) == fc.EINVAL
    assert L.ficoco_window_attention(None, C.byref(_attention()), None) == fc.EINVAL


def test_binding_checks_types_and_shapes():
    c = fc.Cache.empty(1, 4, 16, 2, 64, 3, 2, device="cpu")
    with pytest.raises(TypeError):
        fc.Cache(c.k[:, ::2], c.v, c.k_exp, c.v_exp, c.table, c.len, c.refs)
    with pytest.raises(TypeError):
        fc.Cache(c.k, c.v, c.k_exp, c.v_exp, c.table.long(), c.len, c.refs)
    with pytest.raises(TypeError):
        fc.Cache(c.k, c.v[:, :2], c.k_exp, c.v_exp, c.table, c.len, c.refs)
    assert fc.cache_workspace(c, 3).bytes >= 3 * 2 * 4
    Q = torch.zeros(2, 4, 1, 64, dtype=torch.bfloat16)
    assert fc.attention_workspace(c, Q, torch.zeros_like(Q)).bytes > 0
    with pytest.raises(TypeError):
        fc.attention_workspace(c, Q.float(), torch.zeros_like(Q))
    with pytest.raises(TypeError):
        fc.attention_workspace(c, Q, torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(fc.FicocoError) as e:
        fc.attention_workspace(c, Q, Q)
    assert e.value.code == fc.EINVAL


def test_pages_of_a_call_are_counted_in_32_bits():
    L = fc.lib()
    large = dict(max_pages=1 << 21, page_size=16)
    assert _bytes(L.ficoco_cache_workspace_bytes, C.byref(_cache(**large)), 1023)[0] == fc.OK
    assert _bytes(L.ficoco_cache_workspace_bytes, C.byref(_cache(**large)), 1024)[0] == fc.EUNSUPPORTED
