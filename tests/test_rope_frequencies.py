"""hvd_rope_frequencies (host code) against the formulas, and the layout of the cache operators' structs."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import paper_2606_01019_b200 as H
from paper_2606_01019_b200 import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GEOMETRY = dict(n_q_heads=8, n_kv_heads=2, head_dim=128)


@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (2, 10000.0), (20, 1e6)])
def test_plain_linear_and_base(rot, base):
    i = np.arange(rot // 2)
    w = base ** (-2.0 * i / rot)
    f, m = H.hvd_rope_frequencies(**GEOMETRY, rot_dim=rot, rope_base=base)
    assert np.allclose(f, w, rtol=1e-14) and m == 1.0
    f, m = H.hvd_rope_frequencies(**GEOMETRY, rot_dim=rot, rope_base=base, rope_scaling=H.ROPE_LINEAR, rope_factor=4.0, rope_magnitude=1.5)
    assert np.allclose(f, w / 4, rtol=1e-14) and m == 1.5
    if rot > 2:
        f, _ = H.hvd_rope_frequencies(**GEOMETRY, rot_dim=rot, rope_base=base, rope_scaling=H.ROPE_BASE, rope_factor=8.0)
        assert np.allclose(f[0], 1.0) and np.allclose(f[-1], w[-1] / 8.0, rtol=1e-12)   # the slowest pair stretched by the factor


def test_parts_and_bands():
    L, s, rot, base = 4096.0, 16.0, 128, 10000.0
    w = base ** (-2.0 * np.arange(rot // 2) / rot)
    turns = L * w / (2 * math.pi)
    for kind, lo, hi in ((H.ROPE_PARTS, 1.0, 32.0), (H.ROPE_BANDS, 1.0, 4.0)):
        f, _ = H.hvd_rope_frequencies(**GEOMETRY, rope_scaling=kind, rope_factor=s, rope_original_len=L, rope_low=lo, rope_high=hi)
        ratio = f / w
        assert (np.diff(ratio) <= 1e-12).all()                                           # from 1 down to 1/s
        step = 1.0 if kind == H.ROPE_PARTS else 0.0                                      # the ramp's ends round to whole pairs
        shift = base ** (2.0 * step / rot)
        assert np.allclose(ratio[turns > hi * shift], 1.0) and np.allclose(ratio[turns < lo / shift], 1 / s)
        mid = (turns < hi / shift) & (turns > lo * shift)
        assert mid.any() and ((ratio[mid] < 1) & (ratio[mid] > 1 / s)).all()
    g = np.clip((turns - 1.0) / 3.0, 0, 1)
    assert np.allclose(f, w * g + w / s * (1 - g), rtol=1e-13)


def test_refused_configurations():
    for bad in (dict(rot_dim=3), dict(rot_dim=130), dict(rope_base=0.5), dict(head_dim=20), dict(n_q_heads=3), dict(rope_scaling=7),
                dict(rope_scaling=H.ROPE_LINEAR, rope_factor=0.0), dict(rope_scaling=H.ROPE_BASE, rope_factor=2.0, rot_dim=2),
                dict(rope_scaling=H.ROPE_BANDS, rope_factor=2.0, rope_original_len=10.0, rope_low=4.0, rope_high=1.0), dict(rope_magnitude=-1.0)):
        with pytest.raises(H.HvdError):
            H.hvd_rope_frequencies(**{**GEOMETRY, **bad})


def test_struct_layouts(tmp_path):
    pairs = [("hvd_attn_config", b.HvdAttnConfig), ("hvd_kv_cache", b.HvdKvCache), ("hvd_heads", b.HvdHeads)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "hvd.h"', 'int main(void) {']
    for name, cls in pairs:
        lines.append(f'  printf("%zu", sizeof({name}));' + "".join(f' printf(" %zu", offsetof({name}, {f}));' for f, _ in cls._fields_) + ' printf("\\n");')
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.strip().splitlines()
    for line, (_, cls) in zip(out, pairs):
        assert [int(x) for x in line.split()] == [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
