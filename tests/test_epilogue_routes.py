"""Which kernel a product with something behind it takes for a shape, and into how many slices it is split, on the CPU (host arithmetic for a device of
256 compute units, and of others).  test_gpu_gemm_epilogue.py runs every kernel by its name; these say that the call takes them, that what is
chosen can be launched, and that the workspace depends on sizes and layouts alone."""
import os
import random
import subprocess

import pytest
import torch

import paper_2511_04214_amd as brq

BF16, F32 = torch.bfloat16, torch.float32
LAYOUTS = [("tiled", "tiled"), ("rowmajor", "rowmajor"), ("tiled", "rowmajor"), ("rowmajor", "tiled")]
FORMS = [dict(bias=True), dict(activation="relu"), dict(residual=True), dict(bias=True, activation="gelu", residual=True), dict(activation="silu", out_dtype=BF16),
         dict(bias=True, out_dtype=BF16), dict(residual=True, out_dtype=BF16)]


def choice(M, N, K, layout="tiled", out_dtype=BF16, bias=True, **kw):
    return brq.diag_mxfp4_gemm_epilogue_route(M, N, K, layout, layout, bias=bias, out_dtype=out_dtype, **kw)


# well inside the ranges, and on either side of borders that a comment states with both sides' times
@pytest.mark.parametrize("shape,layout,want", [
    # up to 16 rows
    ((1, 4096, 14336), "tiled", ("few", 1)), ((4, 6144, 4096), "tiled", ("few", 1)), ((16, 4096, 512), "tiled", ("stream", 1)), ((16, 4096, 1024), "tiled", ("few", 1)),
    ((16, 8192, 1024), "tiled", ("stream", 1)), ((16, 8192, 2048), "tiled", ("few", 1)), ((16, 28672, 2048), "tiled", ("stream", 1)), ((16, 28672, 4096), "tiled", ("few", 1)),
    ((16, 28672, 8192), "tiled", ("stream", 1)), ((16, 4096, 1024), "rowmajor", ("stream", 1)), ((16, 4096, 2048), "rowmajor", ("few", 1)),
    ((4, 14336, 4096), "rowmajor", ("few", 1)), ((8, 14336, 4096), "rowmajor", ("stream", 1)), ((4, 70, 1056), "rowmajor", ("skinny", 1)),
    # 17 to 64 rows
    ((48, 4096, 4096), "tiled", ("few", 1)), ((48, 11008, 4096), "tiled", ("few", 1)), ((48, 4096, 11008), "tiled", ("few", 1)), ((24, 4096, 16384), "tiled", ("few", 1)),
    ((64, 4096, 8192), "tiled", ("few", 1)), ((32, 4096, 4096), "rowmajor", ("few", 1)), ((64, 4096, 4096), "rowmajor", ("few", 1)), ((64, 4096, 1024), "rowmajor", ("64x128", 1)),
    ((64, 12289, 4096), "tiled", ("64x128", 1)), ((48, 14336, 4096), "rowmajor", ("64x128", 1)),
    # few tiles and a long K
    ((100, 8192, 28672), "tiled", ("128x128", 3)), ((300, 1288, 8192), "rowmajor", ("64x128", 4)), ((130, 260, 7168), "tiled", ("64x128", 7)), ((17, 8192, 28672), "tiled", ("64x128", 4)),
    # no split, wide tiles, and what no staged kernel takes
    ((4096, 6144, 4096), "tiled", ("128x256", 1)), ((4096, 4096, 14336), "tiled", ("256x256", 1)), ((4096, 6144, 4096), "rowmajor", ("256x256", 1)),
    ((77, 1003, 1056), "rowmajor", ("general", 1)), ((64, 1024, 2080), "rowmajor", ("any_k", 1))])
def test_choice(shape, layout, want):
    assert choice(*shape, layout=layout) == want


# [layout][columns][rows]: the first and last K that the few-rows kernel takes; tiled, and for long K, up to where there are kernels
WINDOWS = {"rowmajor": {4096: {32: (1024, 12288), 48: (1536, 8192), 64: (2048, 4096)}, 8192: {32: (1536, 8192), 48: (2560, 7168), 64: (2560, 4096)},
                        12288: {32: (2560, 12288), 48: (2560, 7168), 64: (3584, 4096)}},
           "tiled": {4096: {32: (512, 16384), 48: (512, 12288), 64: (1024, 8192)}, 8192: {32: (1024, 16384), 48: (1536, 12288), 64: (2048, 8192)},
                     12288: {32: (2048, 12288), 48: (2560, 8192), 64: (3584, 8192)}}}


@pytest.mark.parametrize("layout", ["tiled", "rowmajor"])
def test_few_rows_windows(layout):
    """17 to 64 rows: every K of a window, which is no single size, and none beside it."""
    Ks = sorted({*range(512, 20000, 1024), 1024, 2048, 4096, 5120, 7168, 8192, 12288, 16384})
    for top, by_rows in WINDOWS[layout].items():
        for rows, (first, last) in by_rows.items():
            assert first < last
            for M in (rows - 15, rows):
                for N in (top - 4095, top - 1000, top):
                    for K in Ks:
                        assert (choice(M, N, K, layout=layout)[0] == "few") == (first <= K <= last), (M, N, K)
    for M in (17, 32, 48, 64):
        for K in Ks:
            assert choice(M, 12289, K, layout=layout)[0] != "few"


def test_nothing_behind_is_the_product_alone():
    for shape in ((1, 4096, 4096), (48, 4096, 4096), (100, 8192, 28672), (4096, 6144, 4096)):
        for layout in ("tiled", "rowmajor"):
            assert choice(*shape, layout=layout, bias=False) == (brq.diag_mxfp4_gemm_route(*shape, layout, layout, BF16), 1)


def shapes():
    r = random.Random(5)
    for M in (1, 2, 15, 16, 17, 32, 33, 48, 49, 64, 65, 100, 128, 129, 300, 640, 1000, 2500, 8192):
        for N in (1, 130, 1024, 4096, 4097, 8192, 8193, 12288, 12289, 28672):
            for K in (32, 256, 512, 1024, 1056, 2048, 2560, 4096, 4608, 8192, 8704, 12288, 12800, 16384, 16896, 28672):
                yield M, N, K
    for _ in range(4000):
        yield int(2 ** r.uniform(0, 13.5)), int(2 ** r.uniform(0, 15)), 32 * int(2 ** r.uniform(0, 11))
    for K in (2 ** 24 + 512, 2 ** 25, 2 ** 26 - 512, 2 ** 26, 2 ** 31 - 512):
        for M in (1, 16, 17, 64, 65, 300):
            yield M, 130, K


def test_every_choice_can_be_launched():
    """The call itself answers with an error where the kernel does not take the shape or has no variant for it; slices do not depend on what follows, on the output's type or pitch."""
    seen = set()
    for i, (M, N, K) in enumerate(shapes()):
        cus = (256, 304, 64, 1)[i % 4 if i % 3 == 0 else 0]
        for la, lw in LAYOUTS:
            slices = set()
            for form in FORMS[i % 2:: 2] if i % 5 else FORMS:
                route, n = brq.diag_mxfp4_gemm_epilogue_route(M, N, K, la, lw, ldy=N + i % 9, cus=cus, **form)
                seen.add(route)
                slices.add(n)
                assert n == 1 or route in ("64x128", "128x128")
                assert route != "few" or M <= 64
            assert len(slices) == 1, (M, N, K, la, lw, cus)
    assert seen == set(brq.EPILOGUE_ROUTES)


def test_the_workspace_is_that_of_the_choice(tmp_path):
    """What the library says of the workspace (slices * M * whole quads of N * 4 bytes) against the slices of the choice, for outputs of any type, pitch and address."""
    csrc = os.path.join(os.path.dirname(brq.LIB_PATH), "csrc")
    src, exe = tmp_path / "at.cpp", str(tmp_path / "at")
    src.write_text('''#include <stdio.h>
#include "brq_launch.h"
int main() {
    long split = 0;
    for (int M : {1, 16, 17, 48, 64, 65, 100, 129, 300, 700})
        for (int N : {1, 70, 1288, 4096, 8192, 11008})
            for (int K : {512, 1024, 1056, 2048, 4096, 7168, 8192, 11008, 28672})
                for (int lay = 0; lay < 4; ++lay)
                    for (int form = 0; form < 16; ++form) {
                        const brq::GemmShape asked{M, N, K, (lay & 1) != 0, (lay & 2) != 0, true, N, 0, true};
                        brq::GemmShape g = asked;
                        g.out_bf16 = form & 1;
                        g.ldy = N + (form & 2 ? 5 : 0);
                        g.y = form & 4 ? 48 : 0;
                        g.exponential = form & 8;
                        g.residual = form & 1;
                        const brq::GemmSplit sp = brq::gemm_split(asked, 256);
                        const brq::GemmChoice c = brq::gemm_choice(g, 256);
                        if (c.slices != sp.slices || (c.slices > 1 && c.route != (sp.rows == 64 ? brq::ROUTE_ONE_TILE : brq::ROUTE_ONE_TILE + 1))) return 1;
                        if (brq::split_gemm_workspace(asked, sp) != (c.slices > 1 ? (int64_t)c.slices * M * ((N + 3) / 4 * 16) : 0)) return 2;
                        split += c.slices > 1;
                    }
    printf("%ld\\n", split);
    return split == 0;
}''')
    subprocess.check_call(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__=1", "-isystem/opt/rocm/include", "-I" + csrc, str(src), brq.LIB_PATH, "-o", exe,
                           "-Wl,-rpath," + os.path.dirname(brq.LIB_PATH), "-Wl,-rpath,/opt/rocm/lib", "-Wl,--allow-shlib-undefined"])
    assert int(subprocess.check_output([exe], text=True)) > 0


def test_arguments():
    for bad in (dict(ldy=127), dict(cus=0), dict(cus=1 << 31)):
        with pytest.raises(brq.BrqError) as e:
            choice(4, 128, 512, **bad)
        assert e.value.status == 2
    for shape in ((0, 128, 512), (4, 0, 512), (4, 128, 40), (-1, 128, 512)):
        with pytest.raises(brq.BrqError) as e:
            choice(*shape)
        assert e.value.status == 2
    with pytest.raises(ValueError):
        choice(4, 128, 512, activation="tanh")
    with pytest.raises(ValueError):
        choice(4, 128, 512, layout="columns")
    f = brq.lib().brq_diag_mxfp4_gemm_epilogue_route
    import ctypes
    r, n = ctypes.c_int32(-7), ctypes.c_int32(-7)
    assert f(1, 1, 4, 128, 512, 1, 4, 0, 1, 128, 256, ctypes.byref(r), ctypes.byref(n)) == f(1, 1, 4, 128, 512, 1, -1, 0, 1, 128, 256, ctypes.byref(r), ctypes.byref(n)) == 9
    assert f(1, 1, 4, 128, 512, 1, 0, 0, 1, 128, 256, None, ctypes.byref(n)) == f(1, 1, 4, 128, 512, 1, 0, 0, 1, 128, 256, ctypes.byref(r), None) == 1
    assert (r.value, n.value) == (-7, -7)
