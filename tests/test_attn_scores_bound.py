"""The bound of test_gpu_kv4_attention_scores.py tells sums in 32 bits from sums that keep 14 bits below the largest term (CPU)."""
import torch


def windowed(products, bits):
    """Sums of eight at a time and of the eights, every term cut off `bits` binades below the largest of its sum."""
    def add(x):
        unit = torch.exp2(torch.floor(torch.log2(x.abs().amax(-1, keepdim=True))) - bits)
        return (torch.trunc(x / unit) * unit).sum(-1)
    return add(add(products.unflatten(-1, (-1, 8))))


def test_a_window_of_14_bits_is_seen():
    g = torch.Generator().manual_seed(112)
    small = (2 * torch.randint(0, 8, (200, 128), generator=g) + 1).double() * (1 - 2 * torch.randint(0, 2, (200, 128), generator=g)) * 2.0 ** -10
    at = torch.arange(200)[:, None].remainder(128)
    for cancel in (False, True):
        products = small.scatter(1, at, 256.0)
        if cancel:
            products = products.scatter(1, (at + 1 + at.remainder(127)).remainder(128), -256.0)
        score = products.sum(-1)
        bound = 6 * 2.0 ** -24 * score.abs() + 2.0 ** -18
        assert float(((windowed(products, 14) - score).abs() > bound).double().mean()) > 0.95
        assert torch.equal(windowed(products, 24), score)
