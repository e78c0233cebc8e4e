"""The rotation's part of the ABI without a GPU: layouts of its structs, the table of frequencies, what the binding refuses."""
import ctypes as C
import math
import os
import subprocess
from decimal import Decimal, getcontext

import pytest
import torch

from paper_2411_17686_amd import ficoco as fc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
getcontext().prec = 60
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494")


@pytest.mark.parametrize("name,mirror,packed", [("ficoco_frequencies", fc.FrequenciesProblem, None), ("ficoco_rotary", fc.RotaryProblem, fc._ROTARY),
                                                ("ficoco_rotation", fc.RotationProblem, fc._ROTATION)])
def test_struct_layouts_match_the_header(tmp_path, name, mirror, packed):
    fields = [f[0] for f in mirror._fields_]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ficoco.h"', "int main(void){", 'printf("%%zu\\n", sizeof(%s));' % name]
    lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f in fields] + ["return 0;}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert out[0] == C.sizeof(mirror)
    assert out[1:] == [getattr(mirror, f).offset for f in fields]
    if packed is not None:
        values = [float(3 * i + 1) if t is C.c_float else 3 * i + 1 for i, (_, t) in enumerate(mirror._fields_)]
        assert packed.size == out[0] and packed.pack(*values) == bytes(mirror(*values))


def turns(rot, base, factor=1.0, length=0.0, low=1.0, high=32.0, divisors=None):
    """In 60 digits, as whole numbers of 2^-64 turns."""
    out = []
    for i in range(rot // 2):
        f = (-Decimal(2 * i) / rot * Decimal(base).ln()).exp() / (Decimal(divisors[i]) if divisors else 1)
        s = Decimal(0)
        if length:
            s = min(Decimal(1), max(Decimal(0), (Decimal(length) * f / (2 * PI) - Decimal(low)) / (Decimal(high) - Decimal(low))))
        f *= s + (1 - s) / Decimal(factor)
        part = f / (2 * PI)
        part -= part.to_integral_value(rounding="ROUND_FLOOR")
        out.append(int((part * 2 ** 64).to_integral_value()) % 2 ** 64)
    return out


@pytest.mark.parametrize("kw", [dict(rot=128, base=10000.0), dict(rot=64, base=500000.0, factor=8.0, length=8192.0, low=1.0, high=4.0),
                                dict(rot=2, base=1e6), dict(rot=80, base=10000.0, factor=4.0), dict(rot=512, base=1234.5, factor=32.0, length=4096.0),
                                dict(rot=6, base=100.0, divisors=[1.0, -2.5, 0.125]), dict(rot=0, base=10.0), dict(rot=4, base=0.01)])
def test_frequencies(kw):
    """Extended precision: a relative error of some 2^-61 of at most a tenth of a turn (more where a frequency passes a turn a token)."""
    rot = kw.pop("rot")
    got = [int(x) % 2 ** 64 for x in fc.rotary_turns(rot, **kw)]
    want = turns(rot, **kw)
    assert len(got) == rot // 2
    for g, w in zip(got, want):
        off = (g - w) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= 64


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=514), dict(base=0.0), dict(base=-1.0), dict(base=math.inf), dict(base=math.nan),
                                dict(factor=0.0), dict(factor=math.nan), dict(length=-1.0), dict(length=8.0, low=4.0, high=4.0),
                                dict(length=8.0, low=math.nan), dict(length=math.inf), dict(divisors=[0.0] * 2), dict(divisors=[1.0, math.nan])])
def test_frequencies_refused(kw):
    with pytest.raises(fc.FicocoError) as e:
        fc.rotary_turns(**dict(dict(rot_dim=4), **kw))
    assert e.value.code == fc.EINVAL


def test_null_pointers_are_refused():
    L = fc.lib()
    f = fc.FrequenciesProblem(4, 10.0, 1.0, 0.0, 0.0, 0.0, None)
    assert L.ficoco_rotary_turns(None, None) == fc.EINVAL and L.ficoco_rotary_turns(C.byref(f), None) == fc.EINVAL
    assert L.ficoco_rotate(None, None, None, None) == fc.EINVAL
    assert L.ficoco_cache_append_rotated(None, None, 0, None, None, None, None) == fc.EINVAL


def test_binding_checks_types_and_shapes():
    t = fc.rotary_turns(64)
    w = torch.ones(64)
    for kw in (dict(axis=torch.zeros(31, dtype=torch.uint8)), dict(axis=torch.zeros(32)), dict(q_weight=torch.ones(63)),
               dict(q_weight=w, k_weight=w.bfloat16()), dict(q_weight=torch.ones(2, 64), k_weight=w), dict(q_weight=w.half()),
               dict(k_bias=torch.ones(128)[::2])):
        with pytest.raises(TypeError):
            fc.Rotary(64, t, norm=fc.NORM_RMS, **kw)
    with pytest.raises(TypeError):
        fc.Rotary(64, t.int())
    with pytest.raises(TypeError):
        fc.rotary_turns(8, divisors=[1.0])
    r = fc.Rotary(64, t, norm=fc.NORM_RMS, q_weight=torch.ones(3, 64))
    Q, K = torch.zeros(2, 3, 5, 64), torch.zeros(2, 1, 5, 64)
    assert len(fc._rotation(r, Q, K, Q, K, None, None, None)) == fc._ROTATION.size
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for args in ((torch.zeros(2, 4, 5, 64), None, torch.zeros(2, 4, 5, 64), None, None, None, None), (None, None, None, None, None, None, None),
                 (Q, K, Q, K.bfloat16(), None, None, None), (Q, K[:1], Q, K[:1], None, None, None), (Q, K, Q[:, :2], K, None, None, None),
                 (Q, K, Q, K, i(2, 4), None, None), (Q, K, Q, K, i(5, 2).t(), None, None), (Q, K, Q, K, i(2, 5).long(), None, None),
                 (Q, K, Q, K, None, i(3), None), (Q, K, Q, K, None, None, i(2, 2)[:, 0]), (Q[..., :32], None, Q[..., :32], None, None, None, None)):
        with pytest.raises(TypeError):
            fc._rotation(r, *args)
