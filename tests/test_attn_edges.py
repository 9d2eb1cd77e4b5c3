"""The attention operators where a value, a layout or a step is out of the ordinary.  Plain implementations in 64 bits; bounds
as in test_attn_gpu.py."""
import pytest
import torch

import test_attn_gpu as base
from paper_2405_03133_amd import autograd
from test_attn_gpu import T, freqs, gen, rnd

pytestmark = pytest.mark.gpu


# Head counts that are no multiple of the heads of a load, and tokens on both sides of where one workgroup takes them all.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hkv,D,rot,inter", [(2, 3, 1, 64, 64, False), (500, 3, 1, 64, 64, True), (16, 4, 4, 64, 32, False),
                                                  (300, 5, 2, 128, 128, False), (5, 9, 3, 80, 80, True), (41, 1, 1, 256, 0, False),
                                                  (1200, 8, 8, 8, 0, False), (33, 8, 4, 32, 32, False)])
def test_rope_gradient_without_eps(n, Hq, Hkv, D, rot, inter, dtype, monkeypatch):
    monkeypatch.setattr(base, "EPS", 0.0)
    base.test_rope_gradient(n, Hq, Hkv, D, rot, inter, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_at_any_address(dtype):
    """A gradient that autograd hands over as a contiguous view into a larger one, an element behind a multiple of 16 bytes."""
    t = T[dtype]
    g = gen(31)
    one = torch.ones(1, device="cuda", dtype=t)

    def grads(f, leaves, shift):
        leaves = [x.clone().requires_grad_() for x in leaves]
        loss = 0.0
        for y, c in zip(f(*leaves), factors):
            loss = loss + (torch.cat([one] * shift + [y.reshape(-1)]) * torch.cat([one] * shift + [c])).sum()
        return torch.autograd.grad(loss, leaves)

    n, Hq, Hkv, D = 9, 3, 1, 64
    factors = [rnd(g, n * h * D, dtype=t) for h in (Hq, Hkv)]
    pos, freq = torch.arange(n, device="cuda", dtype=torch.int32), freqs(D)
    leaves = [rnd(g, n, Hq, D, dtype=t), rnd(g, n, Hkv, D, dtype=t), 1 + rnd(g, D, dtype=t) / 4, 1 + rnd(g, D, dtype=t) / 4]
    rope = lambda q, k, wq, wk: autograd.qk_rope(q, k, pos, freq, wq, wk)
    for a, b in zip(grads(rope, leaves, 0), grads(rope, leaves, 1)):
        assert torch.equal(a, b)
    B, L, seg, d, d_ff, E = 1, 128, 64, 128, 256, 4
    factors = [rnd(g, B * L * d, dtype=t)]
    leaves = [rnd(g, B, L, d, dtype=t), rnd(g, d, E, dtype=t) / 8] + [rnd(g, E, *s, dtype=t) / 8 for s in ((d, d_ff), (d, d_ff), (d_ff, d))]
    layer = lambda x, R, Wg, Wu, Wd: [autograd.lory_layer(x, R, Wg, Wu, Wd, seg)]
    for a, b in zip(grads(layer, leaves, 0), grads(layer, leaves, 1)):
        assert torch.equal(a, b)
