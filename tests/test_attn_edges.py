"""The attention operators where a value, a layout or a step is out of the ordinary.  Plain implementations in 64 bits; bounds
as in test_attn_gpu.py."""
import pytest

import test_attn_gpu as base

pytestmark = pytest.mark.gpu


# Head counts that are no multiple of the heads of a load, and tokens on both sides of where one workgroup takes them all.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot,inter", [(2, 3, 1, 64, 64, False), (500, 3, 1, 64, 64, True), (16, 4, 4, 64, 32, False),
                                                  (300, 5, 2, 128, 128, False), (5, 9, 3, 80, 80, True), (41, 1, 1, 256, 0, False),
                                                  (1200, 8, 8, 8, 0, False), (33, 8, 4, 32, 32, False)])
def test_rope_gradient_without_eps(n, Hq, Hkv, D, rot, inter, dtype, monkeypatch):
    monkeypatch.setattr(base, "EPS", 0.0)
    base.test_rope_gradient(n, Hq, Hkv, D, rot, inter, dtype)
