"""mxfp4_gemm_epilogue runs on the kernel and in the slices that its diagnostic names: on operands whose partial sums are not exact, so that
kernels that add in another order differ in bits, the call has the bits of that kernel by name."""
import numpy as np
import pytest
import torch

from gpu_util import to_dev
from test_gpu_layout import to_tiled

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# few rows of either kernel, up to 64 rows, split along K, one tile, wide tiles, any K, what is left
SHAPES = [(1, 700, 1024), (16, 300, 512), (7, 300, 1056), (24, 1500, 4096), (48, 1000, 2048), (64, 520, 4096), (100, 1032, 8192), (300, 1288, 4096), (130, 1000, 7168), (700, 1032, 512),
          (2048, 2048, 1024), (4096, 4096, 512), (64, 1024, 2080), (77, 1003, 1056)]


@pytest.fixture(scope="module")
def brq():
    import paper_2511_04214_amd as b
    b.lib()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return b


def operand(r, rows, K, layout):
    c = r.integers(0, 256, (rows, K // 2), dtype=np.uint8)
    s = r.integers(115, 135, (rows, K // 32), dtype=np.uint8)
    return [to_dev(t) for t in ((c, s) if layout == "rowmajor" else to_tiled(c, s))]


@pytest.mark.parametrize("layout", ["tiled", "rowmajor"])
def test_the_call_takes_what_it_names(brq, layout):
    r, g = np.random.default_rng(7), torch.Generator().manual_seed(7)
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    taken, orders = set(), set()
    for M, N, K in SHAPES:
        a, w = operand(r, M, K, layout), operand(r, N, K, layout)
        bias = torch.randn(N, generator=g).cuda()
        kw = dict(a_layout=layout, w_layout=layout)
        plain = brq.mxfp4_gemm(*a, *w, M=M, N=N, K=K, **kw)
        for act, dt in ((None, F32), ("gelu", BF16)):
            res = torch.randn((M, N), generator=g).to(dt).cuda()
            for b, x in ((bias, None), (bias, res), (None, res)):
                route, slices = brq.diag_mxfp4_gemm_epilogue_route(M, N, K, layout, layout, bias=b is not None, activation=act, residual=x is not None, out_dtype=dt, cus=cus)
                print("case", M, N, K, layout, act, dt, route, slices, flush=True)
                got = brq.mxfp4_gemm_epilogue(*a, *w, bias=b, activation=act, residual=x, out_dtype=dt, M=M, N=N, K=K, **kw)
                want = torch.full((M, N), -7.0, dtype=dt, device="cuda")
                brq.diag_mxfp4_gemm_epilogue_on(route, *a, *w, want, K, bias=b, activation=act, residual=x, slices=slices, **kw)
                assert torch.equal(got, want)
                assert brq.mxfp4_gemm_epilogue_workspace(M, N, K, layout, layout) == (slices * M * ((N + 3) // 4 * 16) if slices > 1 else 0)
                taken.add((route, slices > 1))
                if act is None and x is None:
                    alone = (plain + b).to(dt)
                    orders.add((route in ("few", "skinny") or slices > 1, torch.equal(got, alone)))
    # the kernels that add in the plain product's order have its bits, the few-rows kernel and the slices have not: the bits do tell them apart
    assert (False, True) in orders and (True, False) in orders
    assert {("few", False), ("stream", False)} <= taken and any(split for _, split in taken)
