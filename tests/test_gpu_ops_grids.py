"""Sizes of swam_ops.h that one grid (less than 2^32 threads) does not hold."""
import pytest
import torch

from test_gpu_ops import TYPES, _gpu, check_gemm, contexts, gen  # noqa: F401

pytestmark = pytest.mark.gpu


def room(gb):
    """Skip where the card has less than `gb` GB free."""
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gb * 1e9:
        pytest.skip(f"needs {gb} GB of GPU memory")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("epilogue", ["none", "gated"])
def test_gemm_of_more_columns_than_a_grid_holds(contexts, dtype, epilogue):
    room(48)
    dt, g, n, k = TYPES[dtype], gen(3), (1 << 30) - 1, 16
    w = torch.empty((n, k), dtype=torch.int8, device="cuda")
    for part in w.split(1 << 26):
        part.random_(-128, 128, generator=g)
    a = torch.randint(-128, 128, (1, k), dtype=torch.int8, device="cuda", generator=g)
    sa = torch.rand(1, device="cuda", generator=g) * 0.02 + 1e-3
    sw = torch.rand(n, device="cuda", generator=g).add_(0.1)
    c = torch.full((1, n), float("nan"), dtype=dt, device="cuda")
    b = r = gt = None
    if epilogue == "gated":
        b = torch.empty(n, dtype=dt, device="cuda").uniform_(-1, 1, generator=g)
        r = torch.empty((1, n), dtype=dt, device="cuda").uniform_(-1, 1, generator=g)
        gt = torch.empty(n, device="cuda").uniform_(-1, 1, generator=g)
    contexts[dtype].gemm_i8(a, sa, w, sw, c, bias=b, residual=r, gate=gt)
    assert not any(bool(torch.isnan(part).any()) for part in c.split(1 << 28, 1))
    for lo in (0, (1 << 28) - 4096, (1 << 29) - 20000, (1 << 29) + 4096, 3 << 28, n - 20001):
        at = slice(lo, lo + 20001)
        check_gemm(a, sa, w[at], sw[at], None if b is None else b[at], None if r is None else r[:, at],
                   None if gt is None else gt[at], False, c[:, at])
    del w, c, b, r, gt, sw
    torch.cuda.empty_cache()
