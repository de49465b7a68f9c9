"""Rotation by position of a part of a head leaves the other channels as they are, whatever they hold."""
import math

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan, 3.0e38])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 16), (64, 48), (128, 32), (128, 64), (256, 128), (256, 240)])
def test_channels_behind_the_rotated_ones(D, rot, interleaved, bad):
    g = torch.Generator().manual_seed(61)
    T, H = 5, 3
    x = torch.randn((T, H, D), generator=g)
    angle = torch.rand((10, rot // 2), generator=g) * 6.3
    cos, sin, pos = angle.cos(), angle.sin(), torch.randint(0, 10, (T,), generator=g)
    dev = dict(cos=cos.cuda(), sin=sin.cuda(), positions=pos.cuda(), interleaved=interleaved)
    want = ref.turn(x.double(), cos, sin, pos, interleaved)
    back = ref.turn(x.double(), cos, sin, pos, interleaved, sign=-1.0)
    for c in (rot, D - 1, D - 8):
        y = x.clone()
        y[2, 1, c] = bad
        for got, clean in ((brq.qk_norm_rope(y.cuda(), **dev)[0], want), (brq.qk_norm_rope_backward(x.cuda(), None, y.cuda(), None, **dev)[0], back)):
            got = got.cpu()
            assert torch.equal(got[..., rot:], y[..., rot:]) or (math.isnan(bad) and torch.equal(got[..., rot:].nan_to_num(7.5), y[..., rot:].nan_to_num(7.5)))
            # two products and their sum in 32 bits, of values below 5
            assert ((got[..., :rot].double() - clean[..., :rot]).abs() <= 4 * 2.0 ** -24 * 10).all()


def test_gradients_of_positions_outside_the_tables():
    """NaN in the gradients of their own rows, and in the sums that these are part of."""
    g = torch.Generator().manual_seed(62)
    T, H, D = 9, 3, 64
    x, gr = torch.randn((T, H, D), generator=g).cuda(), torch.randn((T, H, D), generator=g).cuda()
    angle, w = torch.rand((10, D // 2), generator=g) * 6.3, torch.ones(D, device="cuda")
    pos = torch.arange(T)
    a = dict(wq=w, cos=angle.cos().cuda(), sin=angle.sin().cuda())
    want = brq.qk_norm_rope_backward(x, None, gr, None, positions=pos.cuda(), **a)[0]
    pos[3], pos[7] = 10, -1
    dx, _, dw, _ = brq.qk_norm_rope_backward(x, None, gr, None, positions=pos.cuda(), **a)
    out = torch.tensor([3, 7])
    keep = torch.ones(T, dtype=torch.bool)
    keep[out] = False
    assert torch.isnan(dx[out]).all() and torch.equal(dx[keep], want[keep]) and torch.isnan(dw).all()
