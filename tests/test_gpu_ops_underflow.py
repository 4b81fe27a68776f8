"""RMS norm with 8-bit output of rows so small that their float32 squares underflow,
with an eps that does not hide it: y keeps the size of an ordinary row.  The bounds are
those of test_gpu_ops.check_norm (counted roundings; a power of two rounds nothing)."""
import pytest
import torch

from test_gpu_ops import TYPES, _gpu, check_norm, contexts, gen, norm_reference  # noqa: F401

pytestmark = pytest.mark.gpu

# the size of a row's elements; the last rows hold one element, and none
SIZES = [1.0, 1e-15, 1e-18, 2e-19, 1e-20, 1e-21, 1e-22, 1e-23, 1e-26, 1e-30, 1e-34, 1e-37, 1e-39]


def small_rows(d, dt, g, times=1):
    x = torch.randn((len(SIZES), d), device="cuda", generator=g, dtype=torch.float64)
    x = (x * torch.tensor(SIZES, dtype=torch.float64, device="cuda")[:, None]).to(dt)
    lone = torch.zeros((3, d), dtype=dt, device="cuda")
    lone[0, d // 2], lone[1, d - 1] = 1e-25, 2.0 ** -133
    return torch.cat([x, lone]).repeat(times, 1)


def reference(x, r, gain, shift, scale, eps):
    t, y, size = norm_reference(x, r, gain, shift, scale, float(torch.tensor(eps, dtype=torch.float32)))
    # a row of zeros is zeros in front of the shift also without eps
    none = (t == 0).all(1)
    y[none] = 0.0 if shift is None else shift.double()
    size[none] = 0.0 if shift is None else shift.double().abs().amax()
    return t, y, size


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-38, 1e-30, 1e-12])
@pytest.mark.parametrize("d", [5, 64, 130, 1001, 1536, 2049, 2410, 4099, 8192, 9000, 20001])
def test_rows_whose_squares_underflow(contexts, dtype, eps, d):
    dt, g = TYPES[dtype], gen(d)
    for res, mod in ((0, 0), (1, 0), (0, 1)):
        x = small_rows(d, dt, g)
        r = small_rows(d, dt, g) if res else None
        w = (1 + 0.3 * torch.randn(d, device="cuda", generator=g)).to(dt) if mod else None
        sh, sc = (torch.randn((2, d), device="cuda", generator=g) * 0.4).unbind() if mod else (None, None)
        rows = x.shape[0]
        q = torch.full((rows, d), 77, dtype=torch.int8, device="cuda")
        s, total = torch.empty(rows, device="cuda"), torch.empty_like(x)
        contexts[dtype].rms_norm_i8(x, q, s, residual=r, sum_out=total, gain=w, shift=sh, scale=sc, eps=eps)
        check_norm(*reference(x, r, w, sh, sc, eps), q, s, total, dt)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("times,d", [(1700, 101), (500, 1000), (320, 1536), (130, 2410), (80, 8192), (40, 9000)])
def test_small_and_ordinary_rows_in_turn(contexts, dtype, times, d):
    """More rows than run at once, in place: workgroups meet small and ordinary ones in turn."""
    dt, g = TYPES[dtype], gen(times + d)
    x0, r = small_rows(d, dt, g, times), small_rows(d, dt, g, times)
    x0, r = x0[torch.randperm(x0.shape[0], device="cuda", generator=g)], r.flip(0)
    x = x0.clone()
    q = torch.full(x.shape, 77, dtype=torch.int8, device="cuda")
    s = torch.empty(x.shape[0], device="cuda")
    contexts[dtype].rms_norm_i8(x, q, s, residual=r, sum_out=x, eps=0.0)
    check_norm(*reference(x0, r, None, None, None, 0.0), q, s, x, dt)
