"""The 8-bit product on each of its tiles: products for which every one is chosen, ragged
and whole, with every epilogue.  Bounds: test_gpu_ops.check_gemm."""
import ctypes as C
import os

import pytest
import torch

from test_gpu_ops import GEMMS, TYPES, check_gemm, codes, contexts, gen, rows_of, same_outside  # noqa: F401

# more columns or rows than whole tiles, odd and even numbers of 128-code stages, a last stage that
# is not whole; those of test_gpu_ops reach the other tiles
MORE = [(500, 1530, 4112), (500, 1537, 4096), (330, 6150, 1552), (331, 6144, 1536), (2050, 1540, 1936),
        (326, 1536, 6144), (1024, 4096, 1408), (1311, 1030, 1040), (1311, 1030, 912), (1000, 4100, 2064)]


LARGE = [(3472, 1536, 6144), (2001, 6144, 1552), (10160, 1532, 1536), (3474, 6150, 784), (20, 6144, 6160),
         (2600, 4608, 400)]          # of test_gpu_ops.test_gemm_large_products


def test_the_shapes_reach_every_tile():
    """Each tile with rows and columns past whole blocks and a last stage that is not whole,
    those with rings for groups of waves with odd and even numbers of stages (no GPU)."""
    from paper_2609_38984_amd import swam
    if not os.path.exists(swam.LIB_PATH):
        from paper_2609_38984_amd.build import build
        build()
    tile = swam.load_library().swam_gemm_i8_tile
    tile.argtypes, tile.restype = [C.c_int64] * 3, C.c_int
    reached = {}
    for m, n, k in GEMMS + LARGE + MORE:
        reached.setdefault(tile(m, n, k), []).append((m, n, k))
    assert sorted(reached) == list(range(9))
    for t, shapes in reached.items():
        assert any(m % 32 and n % 32 for m, n, _ in shapes), (t, shapes)
        assert any(k % 128 for _, _, k in shapes), (t, shapes)
    for t in (4, 5, 6):
        assert {(k + 127) // 128 % 2 for _, _, k in reached[t]} == {0, 1}, reached[t]
    assert tile(0, 5, 16) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", MORE)
def test_gemm_matches_float64_on_the_tiles_of_middle_sizes(contexts, dtype, m, n, k):
    dt = TYPES[dtype]
    for i, (bias, res, gate, gelu, pad) in enumerate([(0, 0, 0, 0, 0), (1, 0, 0, 1, 16), (1, 1, 1, 0, 0),
                                                      (0, 1, 0, 0, 32)]):
        g = gen(1000 * i + m + n + k)
        a, w = codes(m, k, g, pad), codes(n, k, g, 2 * pad)
        sa = torch.rand(m, device="cuda", generator=g) * 0.02 + 1e-3
        sw = (torch.rand(n, device="cuda", generator=g) + 0.1) * k ** -0.5 / 75
        b = torch.randn(n, device="cuda", generator=g).to(dt) if bias else None
        r = rows_of((m, n), dt, g, pad)[0] if res else None
        gt = torch.randn(n, device="cuda", generator=g) if gate else None
        buf = torch.full((m, n + pad + 1), 7.0, dtype=dt, device="cuda")
        c = buf[:, :n] if pad or n % 8 else torch.full((m, n), 7.0, dtype=dt, device="cuda")
        contexts[dtype].gemm_i8(a, sa, w, sw, c, bias=b, residual=r, gate=gt, gelu=bool(gelu))
        check_gemm(a, sa, w, sw, b, r, gt, gelu, c)
        same_outside(buf, n, 7.0)
        again = torch.empty_like(c)
        contexts[dtype].gemm_i8(a, sa, w, sw, again, bias=b, residual=r, gate=gt, gelu=bool(gelu))
        assert torch.equal(again, c)
