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
