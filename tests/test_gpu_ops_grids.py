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


def test_attention_of_more_tiles_than_a_grid_holds(contexts):
    """float32, 65,535 heads of their own: with one key to a head the output is its value, and
    the normaliser the score."""
    room(235)
    g, heads, n_q, n_seqs, dim = gen(4), 65535, 6309, 64, 64
    q = torch.empty((n_q, heads, dim), device="cuda")
    for part in q.split(256):
        part.uniform_(-1, 1, generator=g)
    k, v = torch.empty((2, n_seqs, heads, dim), device="cuda").uniform_(-1, 1, generator=g)
    o, lse = torch.empty_like(q), torch.empty((n_q, heads), device="cuda")
    for part in o.split(256):
        part.fill_(7.0)
    # one query more than whole tiles of 32 in each sequence: 259 tiles of each head, of which
    # one grid holds 256
    lq = [1 + 32 * (5 * i % 7) for i in range(n_seqs - 1)]
    lq.append(n_q - 5 - sum(lq))
    assert sum((n + 31) // 32 for n in lq) == 259
    cu_q = torch.tensor([0] + lq, device="cuda").cumsum(0).to(torch.int32)
    cu_k = torch.arange(n_seqs + 1, device="cuda", dtype=torch.int32)
    contexts["f32"].cross_attention(q, k, v, o, cu_q=cu_q, cu_k=cu_k, lse=lse)
    at = 0
    for i, n in enumerate(lq):
        for lo in range(at, at + n, 200):
            rows = slice(lo, min(lo + 200, at + n))
            # p is exp2 of a difference of zero up to the rounding of a score below 8: 1 and a sum of
            # itself, divided: 4 roundings of the value
            assert bool(((o[rows] - v[i]).abs() <= 2.0 ** -22 * v[i].abs()).all()), (i, lo)
        first = slice(at, at + 1)
        want = (q[first].double() * k[i].double()).sum(2) / 8
        size = (q[first].double() * k[i].double()).abs().sum(2) / 8
        # 64 products and sums (twice 2^-24 for the matrix unit), the scale, the maximum, the logarithm
        assert bool(((lse[first].double() - want).abs() <= 2 * 80 * 2.0 ** -24 * size + 2.0 ** -20).all()), i
        at += n
    assert bool((o[at:] == 7.0).all())
    del q, o, k, v, lse
    torch.cuda.empty_cache()
