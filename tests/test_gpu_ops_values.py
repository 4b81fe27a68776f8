"""Cross attention where the running maximum moves in every form of it, non-finite values
that are visible, and batches of very unequal lengths; non-finite values through the 8-bit
product's epilogue.  Bounds: test_gpu_ops.check_attention and check_gemm."""
import math

import pytest
import torch

from test_gpu_ops import (TYPES, _gpu, check_attention, check_gemm, codes, contexts, gen, holes, offsets,  # noqa: F401
                          pad_mask, rows_of, run_attention)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# a running maximum that moves
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kvh", [(3, 3), (6, 2), (5, 1)])
@pytest.mark.parametrize("lq", [[1], [70], [300]])
def test_peaked_weights_in_groups_and_under_masks(contexts, dtype, dim, heads, kvh, lq):
    """With one and 70 queries the keys are split, with 300 of several heads not."""
    for i, (scale, std, mask) in enumerate([(0.5, 1.5, None), (1.0, 3.0, holes), (0.125, 6.0, pad_mask)]):
        run_attention(contexts[dtype], TYPES[dtype], lq, [1500], heads, kvh, dim, 21 + i, scale=scale, std=std,
                      mask=mask)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lq,lk", [([2], [3000]), ([40, 9], [700, 1100]), ([2000], [900])])
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_rise_from_tile_to_tile(contexts, dtype, dim, lq, lk, falling):
    """Every tile of a sequence passes the last one's largest score by about 12 (or stays
    below it): a score is the key's place along one direction that all queries share."""
    dt, g = TYPES[dtype], gen(7 + dim)
    n_q, n_k, heads, kvh = sum(lq), sum(lk), 4, 2
    q = torch.randn((n_q, heads, dim), device="cuda", generator=g) * 0.3
    q[:, :, 0] = 4.0
    kv = torch.randn((n_k, 2, kvh, dim), device="cuda", generator=g)
    place = torch.cat([torch.arange(n, device="cuda") for n in lk]) / 64.0
    kv[:, 0, :, 0] = (3.0 * (-place if falling else place))[:, None]
    q, kv = q.to(dt), kv.to(dt)
    k, v = kv[:, 0], kv[:, 1]
    o, lse = torch.full_like(q, 7.0), torch.empty((n_q, heads), device="cuda")
    contexts[dtype].cross_attention(q, k, v, o, cu_q=offsets(lq), cu_k=offsets(lk), lse=lse, scale=1.0)
    check_attention(q, k, v, o, lse, lq, lk, list(range(len(lq))), None, 1.0, o, lse)


# ---------------------------------------------------------------------------
# unequal lengths
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
def test_one_long_prompt_among_short_ones(contexts, dtype, dim):
    run_attention(contexts[dtype], TYPES[dtype], [1] * 64, [5000] + [16] * 63, 4, 2, dim, 5, mask=pad_mask)
    run_attention(contexts[dtype], TYPES[dtype], [1, 200, 3], [9, 3, 4100], 4, 4, dim, 6)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("lk", [[1], [40, 0, 70]])
def test_a_small_part_of_a_large_key_buffer(contexts, dtype, lk):
    """The slices are cut from the buffer's length; most of them are empty here."""
    run_attention(contexts[dtype], TYPES[dtype], [5] * len(lk), lk, 4, 2, 64, 8, behind=12000)


# ---------------------------------------------------------------------------
# non-finite values
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lq,lk", [([3, 1], [2500, 200]), ([150, 33], [300, 65])])
def test_visible_values_that_are_not_finite_stay_in_their_rows(contexts, dtype, dim, lq, lk):
    """A query or key that is NaN, and a score of plus infinity, make the rows of the scores
    that they enter NaN; a value that is not finite makes its column so.  Everything else is as
    without them."""
    dt, g = TYPES[dtype], gen(17 + dim)
    n_q, n_k, heads, kvh = sum(lq), sum(lk), 4, 2
    q, _ = rows_of((n_q, heads, dim), dt, g)
    kv = torch.randn((n_k, 2, kvh, dim), device="cuda", generator=g).to(dt)
    of = [0, 1]
    clean_q, clean_kv = q.clone(), kv.clone()

    def run():
        o, lse = torch.full_like(q, 7.0), torch.full((n_q, heads), 7.0, device="cuda")
        contexts[dtype].cross_attention(q, kv[:, 0], kv[:, 1], o, cu_q=offsets(lq), cu_k=offsets(lk), lse=lse)
        return o, lse

    def check(o, lse, bad):
        """bad: rows and heads that are not finite; the others against the clean inputs."""
        assert bool(torch.isnan(o[bad]).all()) and not bool(torch.isfinite(lse[bad]).any())
        o, lse = o.clone(), lse.clone()
        want, want_lse = torch.empty_like(o), torch.empty_like(lse)
        contexts[dtype].cross_attention(clean_q, clean_kv[:, 0], clean_kv[:, 1], want, cu_q=offsets(lq),
                                        cu_k=offsets(lk), lse=want_lse)
        o[bad], lse[bad] = want[bad], want_lse[bad]
        check_attention(clean_q, clean_kv[:, 0], clean_kv[:, 1], o, lse, lq, lk, of, None, dim ** -0.5, o, lse)

    for value in (float("nan"), float("inf")):
        # one query: a NaN, or scores of both infinities (more than one key)
        q[1, 2, 5] = value
        bad = torch.zeros((n_q, heads), dtype=torch.bool, device="cuda")
        bad[1, 2] = True
        check(*run(), bad)
        q.copy_(clean_q)
        # one key, late in the first sequence, of the second K/V head: with an infinity the
        # queries whose factor is positive score plus infinity (NaN), the others minus infinity:
        # to them the key is hidden
        kv[lk[0] - 40, 0, 1, 3] = value
        bad = torch.zeros((n_q, heads), dtype=torch.bool, device="cuda")
        bad[:lq[0], 2:] = True if math.isnan(value) else clean_q[:lq[0], 2:, 3] > 0
        o, lse = run()
        assert bool(torch.isnan(o[bad]).all()) and bool(torch.isfinite(o[~bad]).all())
        assert bool(torch.isfinite(lse[~bad]).all())
        if math.isnan(value):
            check(o, lse, bad)
        else:
            kv.copy_(clean_kv)
            m = torch.ones(n_k, dtype=torch.bool, device="cuda")
            m[lk[0] - 40] = False
            at = (~bad[:lq[0], 2:]).nonzero()
            want, want_lse = torch.empty_like(o), torch.empty_like(lse)
            contexts[dtype].cross_attention(q, kv[:, 0], kv[:, 1], want, cu_q=offsets(lq), cu_k=offsets(lk),
                                            key_mask=m, lse=want_lse)
            # two results of one formula, each within its bound (bf16: P and o rounded, 2^-8
            # each, on values and sums below 4 in size; lse: see check_attention)
            tol = 2 * (2 * 2.0 ** -8 * 4 if dt == torch.bfloat16 else 1e-4)
            assert bool(((o[at[:, 0], 2 + at[:, 1]] - want[at[:, 0], 2 + at[:, 1]]).abs() <= tol).all())
            assert bool(((lse[at[:, 0], 2 + at[:, 1]] - want_lse[at[:, 0], 2 + at[:, 1]]).abs() <= 1e-4).all())
        kv.copy_(clean_kv)
        # one value of the second sequence, first K/V head
        kv[n_k - 1, 1, 0, 7] = value
        o, lse = run()
        assert not bool(torch.isfinite(o[lq[0]:, :2, 7]).any())
        o[lq[0]:, :2, 7] = 0.0
        v = clean_kv[:, 1].clone()
        v[lk[0]:, 0, 7] = 0.0
        check_attention(clean_q, clean_kv[:, 0], v, o, lse, lq, lk, of, None, dim ** -0.5, o, lse)
        kv.copy_(clean_kv)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n_q,n_k", [(1, 2500), (70, 300), (300, 1000)])
@pytest.mark.parametrize("part", ["first", "last", "all"])
def test_visible_scores_of_minus_infinity_are_as_hidden(contexts, dtype, dim, n_q, n_k, part):
    dt, g, heads = TYPES[dtype], gen(23 + dim), 4
    q, _ = rows_of((n_q, heads, dim), dt, g)
    q[:, :, 0] = 1.0
    k, _ = rows_of((n_k, heads, dim), dt, g)
    v, _ = rows_of((n_k, heads, dim), dt, g)
    seen = torch.ones(n_k, dtype=torch.bool, device="cuda")
    seen[{"first": slice(0, 2 * n_k // 3), "last": slice(n_k // 3, n_k), "all": slice(0, n_k)}[part]] = False
    clean = k.clone()
    k[~seen, :, 0] = -math.inf
    o, lse = torch.full_like(q, 7.0), torch.full((n_q, heads), 7.0, device="cuda")
    contexts[dtype].cross_attention(q, k, v, o, lse=lse)
    check_attention(q, clean, v, o, lse, [n_q], [n_k], [0], seen, dim ** -0.5, o, lse)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(1, 40, 48), (130, 264, 272), (700, 1540, 528)])
def test_infinities_through_the_epilogue(contexts, dtype, m, n, k):
    """A bias or residual that is not finite goes through the formula into its own column or
    element (GELU of minus infinity is NaN: 0 times infinity), and a zero scale beside them
    gives the bias alone."""
    dt, g = TYPES[dtype], gen(m + n)
    a, w = codes(m, k, g), codes(n, k, g)
    sa = torch.rand(m, device="cuda", generator=g) * 0.02 + 1e-3
    sw = (torch.rand(n, device="cuda", generator=g) + 0.1) * k ** -0.5 / 75
    b, gate = torch.randn(n, device="cuda", generator=g).to(dt), torch.randn(n, device="cuda", generator=g)
    b[3], b[8], b[n - 1], b[11] = math.inf, -math.inf, math.nan, 3e38
    b[12], sw[12] = -3e38, 0.0
    odd = torch.zeros(n, dtype=torch.bool, device="cuda")
    odd[[3, 8, n - 1, 11, 12]] = True
    r = rows_of((m, n), dt, g)[0]
    r[0, 20], r[m - 1, 21] = math.inf, -math.inf
    c = torch.empty((m, n), dtype=dt, device="cuda")
    contexts[dtype].gemm_i8(a, sa, w, sw, c, bias=b, gelu=True)
    assert bool((c[:, 3] == math.inf).all()) and bool(torch.isnan(c[:, 8]).all()) and bool(torch.isnan(c[:, n - 1]).all())
    assert bool((c[:, 11].double() / 3e38 - 1.0).abs().amax() < 0.01) and bool((c[:, 12] == 0).all())
    keep = ~odd
    check_gemm(a, sa, w[keep], sw[keep], b[keep], None, None, True, c[:, keep])
    contexts[dtype].gemm_i8(a, sa, w, sw, c, bias=b, residual=r, gate=gate)
    assert bool((c[:, 3] == math.copysign(math.inf, float(gate[3]))).all()) and bool(torch.isnan(c[:, n - 1]).all())
    assert float(c[0, 20]) == math.inf and float(c[m - 1, 21]) == -math.inf
    keep[20:22] = False
    check_gemm(a, sa, w[keep], sw[keep], b[keep], r[:, keep], gate[keep], False, c[:, keep])
