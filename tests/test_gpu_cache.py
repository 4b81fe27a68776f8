"""The operators of swam_cache.h on the GPU against plain float64 forms, at the sizes,
strides, pages and masks where they can go wrong.  u = 2^-24 is half a step of float32 and h
that of the storage type (bf16: 2^-8); every bound below is the count of such roundings on
the way, written beside it."""
import math

import pytest
import torch

import workload as W
from test_gpu_ops import HALF, TYPES, U, _gpu, gen, offsets, rows_of, same_outside  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def contexts():
    from paper_2609_38984_amd import swam
    return {t: swam.Context(W.preset(2).replace(dtype=t, n_blocks=1)) for t in TYPES}


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------
def post64(x, pos, norm, eps, gain, freq, half, mag):
    """Norm and rotation of heads [rows][heads][dim] in float64, and the bound of float32
    work on it (before the rounding to storage)."""
    y = x.double()
    dim = y.shape[-1]
    # sum of squares: 8 products in a chain and 6 exchanges, 7 u under the root; the mean, eps and
    # the root 3 u; two products: 12 u
    rel = 0.0
    if norm:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
        y = torch.where(x.double().abs().amax(-1, keepdim=True) > 0, y, torch.zeros_like(y))
        rel = 12 * U
        if gain is not None:
            y = y * gain.double()
            rel += U
    err = rel * y.abs()
    n = 2 * len(freq)
    if n:
        f = freq.double()
        angle = pos.double()[:, None] * f
        # the turns: two roundings in float64 here and three there, one to float32 of at most half
        # a turn (pi u), sine and cosine 4 u, times m: 9 u
        a_err = 2.0 ** -50 * angle.abs() + 9 * U
        c, s, a_err = (t[:, None] for t in (torch.cos(angle), torch.sin(angle), a_err))
        i = torch.arange(n // 2, device=x.device)
        first, second = (i, i + n // 2) if half else (2 * i, 2 * i + 1)
        a, b = y[..., first], y[..., second]
        ea, eb = err[..., first], err[..., second]
        out, oerr = y.clone(), err.clone()
        out[..., first], out[..., second] = mag * (a * c - b * s), mag * (a * s + b * c)
        # both products and the sum: 3 u of the larger terms
        both = abs(mag) * ((a_err + 3 * U) * (a.abs() + b.abs()) + ea + eb)
        oerr[..., first] = both
        oerr[..., second] = both
        y, err = out, oerr
    return y, err


def check_close(got, want, err, h):
    # below 2^-126 the steps of both types stay what they are there (bf16 2^-133, float32 2^-149),
    # and half of one is h 2^-126
    err = err + h * (want.abs() + err) + h * 2.0 ** -126 + 2.0 ** -149
    off = (got.double() - want).abs()
    assert bool((off <= err).all()), float((off / err).max())


def freq_of(rot, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")


def make_post(dt, dim, rot, half, norm=True, gain=True, mag=1.0, eps=1e-6, seed=0):
    from paper_2609_38984_amd import swam
    g = gen(900 + seed)
    gains = [(1 + 0.3 * torch.randn(dim, device="cuda", generator=g)).to(dt) if norm and gain else None for _ in range(2)]
    freq = freq_of(rot) if rot else torch.zeros(0, dtype=torch.float64, device="cuda")
    rope = swam.Rope(freq, "half" if half else "interleaved", mag) if rot else None
    return swam.QkPost(norm=norm, eps=eps, q_gain=gains[0], k_gain=gains[1], rope=rope), gains, freq


HEAD_SHAPES = [(1, 1, 1, 8, 8), (3, 2, 1, 16, 10), (5, 3, 3, 24, 24), (7, 24, 24, 64, 64), (2, 5, 1, 64, 32),
               (9, 4, 2, 80, 20), (4, 6, 2, 96, 96), (1, 16, 4, 128, 64), (33, 7, 1, 128, 128), (6, 2, 2, 128, 42),
               (3, 3, 1, 200, 6), (5, 2, 1, 256, 256), (2, 1, 1, 512, 384), (1500, 3, 2, 64, 64), (5000, 1, 1, 128, 128)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("rows,heads,kvh,dim,rot", HEAD_SHAPES)
def test_norm_and_rotation_match_float64(contexts, dtype, half, rows, heads, kvh, dim, rot):
    dt = TYPES[dtype]
    for n, (norm, gain, mag, pad, rotate) in enumerate([(True, True, 1.0, 0, True), (True, False, 1.25, 8, True),
                                                        (False, False, 1.0, 16, True), (True, True, 1.0, 8, False)]):
        g = gen(10 * n + rows + dim)
        post, gains, freq = make_post(dt, dim, rot if rotate else 0, half, norm, gain, mag, seed=n)
        # q, k and v of a row side by side, as a projection leaves them
        x = torch.randn((rows, (heads + 2 * kvh) * dim + pad), device="cuda", generator=g).to(dt)
        q = x[:, :heads * dim].unflatten(1, (heads, dim))
        k = x[:, heads * dim:(heads + kvh) * dim].unflatten(1, (kvh, dim))
        before = x.clone()
        pos = torch.randint(0, 50000, (rows,), device="cuda", generator=g).to(torch.int32) if n != 1 else None
        at = pos if pos is not None else torch.arange(rows, device="cuda")
        qo, qbuf = rows_of((rows, heads, dim), dt, g, pad, fill=7.0)
        ko, kbuf = rows_of((rows, kvh, dim), dt, g, pad, fill=7.0)
        contexts[dtype].qk_norm_rope(q, k, post, pos=pos, q_out=qo, k_out=ko)
        for got, src, gain_t in ((qo, q, gains[0]), (ko, k, gains[1])):
            want, err = post64(src, at, norm, 1e-6, gain_t, freq, half, mag)
            check_close(got, want, err, HALF[dt])
        assert torch.equal(x, before)
        same_outside(qbuf, heads * dim, 7.0)
        same_outside(kbuf, kvh * dim, 7.0)
        # in place, and one of the two alone: the same bits, v and padding untouched
        contexts[dtype].qk_norm_rope(q, k, post, pos=pos)
        assert torch.equal(q, qo) and torch.equal(k, ko)
        assert torch.equal(x[:, (heads + kvh) * dim:], before[:, (heads + kvh) * dim:])
        y = before.clone()
        contexts[dtype].qk_norm_rope(y[:, :heads * dim].unflatten(1, (heads, dim)), None, post, pos=pos)
        assert torch.equal(y[:, :heads * dim], x[:, :heads * dim]) and torch.equal(y[:, heads * dim:], before[:, heads * dim:])
        y = before.clone()
        contexts[dtype].qk_norm_rope(None, y[:, heads * dim:(heads + kvh) * dim].unflatten(1, (kvh, dim)), post, pos=pos)
        assert torch.equal(y[:, heads * dim:], x[:, heads * dim:]) and torch.equal(y[:, :heads * dim], before[:, :heads * dim])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("half", [False, True])
def test_far_and_negative_positions(contexts, dtype, half):
    """Positions to the ends of int32: an angle in float32 would be off by radians."""
    dt, g = TYPES[dtype], gen(5)
    pos = torch.tensor([0, 1, -1, 17472, 1 << 20, -(1 << 20), (1 << 24) + 1, (1 << 30) + 12345, (1 << 31) - 1, -(1 << 31)],
                       device="cuda").to(torch.int32)
    post, gains, freq = make_post(dt, 64, 64, half)
    q, _ = rows_of((10, 3, 64), dt, g)
    qo = torch.empty_like(q)
    contexts[dtype].qk_norm_rope(q, None, post, pos=pos, q_out=qo)
    want, err = post64(q, pos, True, 1e-6, gains[0], freq, half, 1.0)
    check_close(qo, want, err, HALF[dt])
    # position 0 rotates nothing
    plain, _, _ = make_post(dt, 64, 0, half)
    other = torch.empty_like(q)
    contexts[dtype].qk_norm_rope(q, None, plain, q_out=other)
    assert torch.equal(other[0], qo[0])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 64), (80, 20), (128, 52)])
def test_heads_that_are_zero_tiny_huge_or_not_finite(contexts, dtype, half, dim, rot):
    dt, g = TYPES[dtype], gen(7)
    x, _ = rows_of((9, 4, dim), dt, g)
    x[0, 1] = 0.0
    x[1, 2] *= 1e-22                                   # squares underflow float32
    x[2, 0] = (x[2, 0].double() * 2.0 ** -130).to(dt)   # subnormal
    x[3, 3] = (x[3, 3].double() * 1e30).to(dt)          # squares overflow
    x[4, 1] = 3e38
    x[5, 2, dim - 1] = float("nan")
    x[6, 0, 1] = float("inf")
    x[7, 1] *= 1e-12
    for eps in (0.0, 1e-6, 1e-35):
        post, gains, freq = make_post(dt, dim, rot, half, eps=eps)
        y = torch.empty_like(x)
        contexts[dtype].qk_norm_rope(x, None, post, q_out=y)
        bad = torch.zeros((9, 4), dtype=torch.bool, device="cuda")
        bad[5, 2] = bad[6, 0] = True
        at = torch.arange(9, device="cuda")
        want, err = post64(x, at, True, eps, gains[0], freq, half, 1.0)
        check_close(y[~bad], want[~bad], err[~bad] + 2.0 ** -140, HALF[dt])
        assert bool(torch.isnan(y[5, 2]).all()) and bool(torch.isnan(y[6, 0, 1]))
        assert bool((y[0, 1] == 0).all())
    # without the norm a value that is not finite stays in its pair
    post, _, freq = make_post(dt, dim, rot, half, norm=False)
    y = torch.empty_like(x)
    contexts[dtype].qk_norm_rope(x, None, post, q_out=y)
    partner = (1 + rot // 2 if half else 0)
    odd = ~torch.isfinite(y)
    hit = torch.zeros_like(odd)
    hit[5, 2, dim - 1] = True
    hit[6, 0, 1] = hit[6, 0, partner] = True
    if rot == dim:
        hit[5, 2, dim - 1 - (rot // 2 if half else 1)] = True
    assert torch.equal(odd & (x.abs() < 2e38), hit & (x.abs() < 2e38))


# ---------------------------------------------------------------------------
# the cache
# ---------------------------------------------------------------------------
class Paged:
    """A cache with pages in no order, NaN wherever nothing was put."""

    def __init__(self, dt, lengths, room, page, kvh, dim, seed=0, by_head=True, spare=3, joint=False, fill=float("nan")):
        from paper_2609_38984_amd import swam
        g = gen(1000 + seed)
        held = [-(-r // page) for r in room]
        n = sum(held) + spare
        perm = torch.randperm(n, device="cuda", generator=g).tolist()
        width = max(held + [1])
        shape = (n, kvh, page, dim) if by_head else (n, page, kvh, dim)
        if joint:
            both = torch.full((n, 2) + shape[1:], fill, dtype=dt, device="cuda")
            k, v = both[:, 0], both[:, 1]
        else:
            k, v = (torch.full(shape, fill, dtype=dt, device="cuda") for _ in range(2))
        self.k, self.v = (t.transpose(1, 2) if by_head else t for t in (k, v))
        rows, at = [], 0
        for h in held:
            rows.append(perm[at:at + h] + [-1] * (width - h))
            at += h
        self.table = torch.tensor(rows, dtype=torch.int32, device="cuda")
        self.length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.page, self.lengths, self.dim, self.kvh = page, list(lengths), dim, kvh
        self.c = swam.Cache(self.k, self.v, self.table, self.length)

    def where(self, s, j):
        return self.table[s].long()[j // self.page], j % self.page

    def put(self, s, lo, hi, g, std=1.0):
        j = torch.arange(lo, hi, device="cuda")
        p, t = self.where(s, j)
        for c in (self.k, self.v):
            c[p, t] = (torch.randn((hi - lo, self.kvh, self.dim), device="cuda", generator=g) * std).to(c.dtype)


APPENDS = {
    "one_token": ([1], [0], 16, 4, 2, 64), "one_late": ([1], [133], 16, 6, 3, 128), "tokens_of_5": ([1] * 5, [0, 15, 16, 17, 300], 16, 2, 2, 64),
    "empty_among": ([0, 9, 0, 33], [5, 7, 0, 31], 8, 3, 1, 64), "page_ends": ([8, 16, 24], [8, 0, 4], 8, 2, 1, 128),
    "long": ([700], [90], 64, 8, 8, 64), "ragged": ([300, 1, 77, 129], [1000, 3, 0, 255], 32, 7, 1, 128),
    "large_page": ([500, 40], [0, 1000], 1024, 4, 4, 64), "many": ([(3 * i) % 5 for i in range(300)], [(7 * i) % 40 for i in range(300)], 16, 2, 1, 64),
    "thousand": ([1] * 1024, [(11 * i) % 50 for i in range(1024)], 8, 2, 2, 64),
}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("name", list(APPENDS))
def test_append_matches_float64(contexts, dtype, half, name):
    new, old, page, heads, kvh, dim = APPENDS[name]
    dt = TYPES[dtype]
    for n, (by_head, joint, norm, rot, own_pos, with_q, pad) in enumerate([
            (True, False, True, dim, False, True, 0), (False, False, True, dim // 2, True, True, 8),
            (False, True, False, 0, False, False, 16), (True, True, True, 10, False, True, 8)]):
        g = gen(n + len(name))
        c = Paged(dt, old, [a + b for a, b in zip(new, old)], page, kvh, dim, n, by_head, joint=joint, fill=5.0)
        post, gains, freq = make_post(dt, dim, rot, half, norm, seed=n)
        behind, rows = 3, sum(new) + 3
        x = torch.randn((rows, (heads + 2 * kvh) * dim + pad), device="cuda", generator=g).to(dt)
        q, k, v = (t.unflatten(1, (-1, dim)) for t in x[:, :(heads + 2 * kvh) * dim].split((heads * dim, kvh * dim, kvh * dim), 1))
        pos = torch.randint(-9, 9999, (rows,), device="cuda", generator=g).to(torch.int32) if own_pos else None
        qo = torch.full((rows, heads, dim), 9.0, dtype=dt, device="cuda")
        want_k, want_v = c.k.double(), c.v.double()
        err_k = torch.zeros_like(want_k)
        contexts[dtype].cache_append(c.c, k, v, cu=offsets(new), q=q if with_q else None, q_out=qo if with_q else None,
                                     post=post if norm or rot else None, pos=pos)
        at = 0
        for s, m in enumerate(new):
            r = slice(at, at + m)
            at += m
            j = torch.arange(old[s], old[s] + m, device="cuda")
            p, t = c.where(s, j)
            a = pos[r] if own_pos else j
            want_k[p, t], err_k[p, t] = post64(k[r], a, norm, 1e-6, gains[1], freq, half, 1.0)
            want_v[p, t] = v[r].double()
            if with_q:
                check_close(qo[r], *post64(q[r], a, norm, 1e-6, gains[0], freq, half, 1.0), HALF[dt])
        check_close(c.k, want_k, err_k, HALF[dt] if norm or rot else 0.0)
        # values, and what nothing was appended to, are as they were
        assert torch.equal(c.v.double(), want_v)
        assert torch.equal(c.k[err_k == 0].double(), want_k[err_k == 0])
        assert bool((qo[rows - behind:] == 9.0).all())
        if with_q:
            # in place
            k2, v2, x2 = c.k.clone(), c.v.clone(), x.clone()
            q2 = x2[:, :heads * dim].unflatten(1, (heads, dim))
            contexts[dtype].cache_append(c.c, k, v, cu=offsets(new), q=q2, post=post if norm or rot else None, pos=pos)
            assert torch.equal(q2[:sum(new)], qo[:sum(new)]) and torch.equal(x2[sum(new):], x[sum(new):])
            assert torch.equal(c.k, k2) and torch.equal(c.v, v2)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_append_without_a_place(contexts, dtype):
    """Table entries outside the pages, tokens past the table, lengths outside it: nothing is
    written for them, their queries are."""
    dt, g = TYPES[dtype], gen(3)
    c = Paged(dt, [4, 30, -5, 1 << 30], [64] * 4, 8, 2, 64, fill=5.0)
    c.table[0, 1], c.table[0, 2], c.table[1, 4] = -7, len(c.k), 1 << 30
    new = [20, 50, 6, 4]
    q, k, v = (torch.randn((80, n, 64), device="cuda", generator=g).to(dt) for n in (4, 2, 2))
    want_k, want_v = c.k.clone(), c.v.clone()
    qo = torch.full_like(q, 9.0)
    contexts[dtype].cache_append(c.c, k, v, cu=offsets(new), q=q, q_out=qo)
    start = [4, 30, 0, 64]
    at = 0
    for s, n in enumerate(new):
        for i in range(n):
            j = start[s] + i
            if j < 64 and 0 <= int(c.table[s, j // 8]) < len(c.k):
                want_k[int(c.table[s, j // 8]), j % 8], want_v[int(c.table[s, j // 8]), j % 8] = k[at + i], v[at + i]
        at += n
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v) and torch.equal(qo, q)
    # offsets outside the rows end at them, falling ones make empty sequences
    cu = torch.tensor([-9, 20, 20, 15, 1 << 30], dtype=torch.int32, device="cuda")
    qo.fill_(9.0)
    contexts[dtype].cache_append(c.c, k, v, cu=cu, q=q, q_out=qo)
    torch.cuda.synchronize()


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_cache_attention(c, q, o, lse, new, causal, window, scale, o_before, lse_before, places=None):
    """places(s): the keys of sequence s that have a place (default: all)."""
    heads, dim = q.shape[1:]
    group, h, at = heads // c.kvh, HALF[q.dtype], 0
    for s, n in enumerate(new):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        total = c.lengths[s] + n
        j = torch.arange(total, device="cuda") if places is None else places(s, total)
        i = torch.arange(c.lengths[s], total, device="cuda")[:, None]
        see = torch.ones((n, j.numel()), dtype=torch.bool, device="cuda")
        if causal:
            see &= j <= i
        if window:
            see &= i - j < window
        p, t = c.where(s, j)
        # (what a row does not see may hold anything)
        some = see.any(0)
        k, v = c.k[p, t].double(), c.v[p, t].double()
        k[~some], v[~some] = 0.0, 0.0
        for hd in range(heads):
            kj, vj, qj = k[:, hd // group], v[:, hd // group], q[rows, hd].double()
            x = (qj @ kj.t().contiguous() * scale).masked_fill(~see, -math.inf)
            m = x.amax(1, keepdim=True) if j.numel() else torch.full((n, 1), -math.inf, device="cuda", dtype=torch.float64)
            live = (m > -math.inf)[:, 0]
            assert bool((o[rows, hd][~live] == 0).all())
            assert lse is None or bool((lse[rows, hd][~live] == -math.inf).all())
            if not bool(live.any()):
                continue
            x, m = x[live], m[live]
            w = torch.exp(x - m)
            l = w.sum(1, keepdim=True)
            want, wl, size = (w / l) @ vj, (m + torch.log(l))[:, 0], (w / l) @ vj.abs()
            qk = ((qj[live].abs() @ kj.abs().t().contiguous()) * scale).masked_fill(~see[live], 0.0).amax(1)
            # a logit: dim products and sums in float32 (twice u for the matrix unit), the
            # scale and the maximum; then exp2.  Sums over the keys: one rounding per key.
            lerr = (2 * (dim + 8) * U * qk + 8 * U * wl.abs())[:, None]
            sums = (j.numel() + 16) * U
            err = (h + 2 * lerr + 2 * sums) * 1.01 * size
            err = err + (h + 4 * U) * (want.abs() + err)
            off = (o[rows, hd][live].double() - want).abs()
            assert bool((off <= err).all()), (s, hd, float((off / err).max()))
            if lse is not None:
                lse_err = 1.01 * (lerr[:, 0] + sums) + 4 * U * wl.abs()
                assert bool(((lse[rows, hd][live].double() - wl).abs() <= lse_err).all()), (s, hd)
    assert torch.equal(o[at:], o_before[at:])
    assert lse is None or torch.equal(lse[at:], lse_before[at:])


def run_cache_attention(ctx, dt, new, old, heads, kvh, dim, page, causal=True, window=0, seed=0, by_head=True, joint=False,
                        pad=0, std=1.0, scale=None, want_lse=True, behind=3, change=None, places=None):
    g = gen(seed)
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], page, kvh, dim, seed, by_head, joint=joint)
    for s in range(len(new)):
        c.put(s, 0, old[s] + new[s], g, std)
    if change is not None:
        change(c)
    rows = sum(new) + behind
    q, _ = rows_of((rows, heads, dim), dt, g, pad, std)
    o, obuf = rows_of((rows, heads, dim), dt, g, pad, fill=7.0)
    lse = torch.randn((rows, heads), device="cuda", generator=g) if want_lse else None
    before = o.clone(), None if lse is None else lse.clone()
    ctx.cache_attention(c.c, q, o, cu=offsets(new), causal=causal, window=window, scale=scale, lse=lse)
    check_cache_attention(c, q, o, lse, new, causal, window, dim ** -0.5 if scale is None else scale, *before, places=places)
    same_outside(obuf, heads * dim, 7.0)
    return o


SHAPES = {
    "one_of_one": ([1], [0], 1, 1, 64, 16), "one_long": ([1], [5000], 3, 3, 64, 16), "one_group": ([1], [1536], 14, 2, 128, 64),
    "tokens_of_8": ([1] * 8, [700] * 8, 4, 4, 64, 32), "prefill": ([326], [0], 5, 5, 64, 16),
    "odd": ([129, 1, 63], [65, 64, 1], 3, 1, 64, 8), "empty_among": ([0, 5, 0, 40], [3, 0, 9, 130], 2, 2, 64, 16),
    "group_7": ([37, 70], [200, 31], 7, 1, 64, 128), "wide_head": ([300], [513], 4, 2, 128, 16),
    "wide_odd": ([31, 33, 257], [129, 63, 1], 6, 3, 128, 8), "many_tiles": ([1000], [300], 4, 4, 64, 64),
    "sixty_four": ([3] * 64, [17] * 64, 2, 1, 64, 16), "few_long": ([9, 20], [3001, 2000], 2, 2, 128, 256),
    "small_group_long": ([6], [9999], 8, 4, 64, 16), "mid_batch": ([200, 150, 40], [600, 512, 700], 8, 8, 64, 32),
    "unequal": ([1] * 16, [6000] + [5] * 15, 4, 1, 128, 16), "mixed": ([400, 1, 1, 1], [50, 3000, 10, 900], 6, 2, 64, 64),
    "huge_page": ([70, 1], [900, 5000], 3, 3, 64, 4096), "two_hundred": ([(i * 7) % 4 for i in range(200)], [(i * 13) % 90 for i in range(200)], 2, 1, 64, 8),
}


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention_matches_float64(contexts, dtype, causal, name):
    for i, (window, pad, by_head, joint, want_lse) in enumerate([(0, 0, True, False, True), (90, 8, False, False, True),
                                                                 (1, 0, False, True, False)]):
        run_cache_attention(contexts[dtype], TYPES[dtype], *SHAPES[name], causal=causal, window=window, seed=10 * i + len(name),
                            by_head=by_head, joint=joint, pad=pad, want_lse=want_lse)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("window", [2, 63, 64, 65, 500, (1 << 31) - 1])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(contexts, dtype, window, causal):
    run_cache_attention(contexts[dtype], TYPES[dtype], [150, 3], [1000, 2500], 4, 2, 64, 16, causal, window, 3)
    run_cache_attention(contexts[dtype], TYPES[dtype], [1, 700], [4000, 0], 3, 1, 128, 32, causal, window, 4)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("scale,std", [(0.5, 1.5), (1.0, 3.0), (1e-3, 1.0), (0.125, 6.0)])
@pytest.mark.parametrize("new,old", [([1], [1500]), ([70], [1400]), ([300, 2], [20, 3000])])
@pytest.mark.parametrize("dim", [64, 128])
def test_peaked_and_flat_weights(contexts, dtype, scale, std, new, old, dim):
    """The running maximum moves again and again, or never."""
    run_cache_attention(contexts[dtype], TYPES[dtype], new, old, 6, 3, dim, 16, seed=21, scale=scale, std=std)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_scores_that_rise_from_tile_to_tile(contexts, dtype, falling, dim):
    dt, g = TYPES[dtype], gen(7)
    new, old = [200, 1], [500, 2500]
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], 16, 2, dim)
    for s in range(2):
        c.put(s, 0, old[s] + new[s], g)
        j = torch.arange(old[s] + new[s], device="cuda")
        p, t = c.where(s, j)
        c.k[p, t, :, 0] = (3.0 * (-j if falling else j) / 64.0)[:, None].to(dt)
    q = torch.randn((201, 4, dim), device="cuda", generator=g) * 0.3
    q[:, :, 0] = 4.0
    q = q.to(dt)
    o, lse = torch.empty_like(q), torch.empty((201, 4), device="cuda")
    contexts[dtype].cache_attention(c.c, q, o, cu=offsets(new), scale=1.0, lse=lse)
    check_cache_attention(c, q, o, lse, new, True, 0, 1.0, o, lse)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new,old,page", [([1, 1, 1], [900, 70, 30], 16), ([150, 40, 9], [300, 70, 0], 8), ([1, 200], [5000, 64], 64)])
def test_pages_that_hold_nothing(contexts, dtype, causal, new, old, page):
    """Entries outside the cache at the start, inside and at the end of a tile, and for a
    whole sequence: their keys are not seen, and a row with no other key is zeros."""
    lost = [[0, 2, 3, 17], [1], None]

    def change(c):
        for s in range(len(new)):
            drop = lost[s]
            idx = torch.arange(c.table.shape[1], device="cuda") if drop is None else \
                torch.tensor([d for d in drop if d < c.table.shape[1]], device="cuda")
            c.table_before = getattr(c, "table_before", c.table.clone())
            c.table[s, idx] = torch.tensor([-1, len(c.k), 1 << 30, -(1 << 31)], device="cuda").to(torch.int32)[idx % 4]
        c.where = lambda s, j: (c.table_before[s].long()[j // c.page], j % c.page)

    def places(s, total):
        j = torch.arange(total, device="cuda")
        if lost[s] is None:
            return j[:0]
        keep = torch.ones(total, dtype=torch.bool, device="cuda")
        for d in lost[s]:
            keep &= j // page != d
        return j[keep]

    for dim in (64, 128):
        run_cache_attention(contexts[dtype], TYPES[dtype], new, old, 4, 2, dim, page, causal, seed=5, change=change, places=places)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_lengths_and_offsets_are_clamped(contexts, dtype):
    dt, g = TYPES[dtype], gen(9)
    c = Paged(dt, [0, 0], [64, 64], 8, 2, 64)
    for s in range(2):
        c.put(s, 0, 64, g)
    q, _ = rows_of((12, 2, 64), dt, g)
    o = torch.full_like(q, 7.0)
    lse = torch.full((12, 2), 7.0, device="cuda")
    # a negative length is none; one past the table leaves every key of it, all before the chunk
    c.length.copy_(torch.tensor([-8, 1 << 30], device="cuda"))
    cu = torch.tensor([-3, 8, 1 << 30], dtype=torch.int32, device="cuda")
    contexts[dtype].cache_attention(c.c, q, o, cu=cu, lse=lse)
    c.lengths = [0, 64]
    a = o.clone()
    check_cache_attention(c, q[:8], o[:8], lse[:8], [8], True, 0, 0.125, o[:8], lse[:8])
    # the second sequence by hand: 64 keys for each of its 4 tokens
    j = torch.arange(64, device="cuda")
    p, t = c.where(1, j)
    for h in range(2):
        x = q[8:, h].double() @ c.k[p, t, h].double().t().contiguous() * 0.125
        want = torch.softmax(x, 1) @ c.v[p, t, h].double()
        assert bool(((o[8:, h].double() - want).abs() <= 3 * HALF[dt] * c.v[p, t, h].double().abs().max()).all())
    # a sequence without a place at all
    from paper_2609_38984_amd import swam
    none = swam.Cache(c.k, c.v, c.table[:, :0], c.length)
    contexts[dtype].cache_attention(none, q, o, cu=cu, lse=lse)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())
    empty = swam.Cache(c.k[:0], c.v[:0], c.table, c.length)
    o.fill_(7.0)
    contexts[dtype].cache_attention(empty, q, o, cu=cu)
    assert bool((o == 0).all())
    # rows outside every sequence
    o.fill_(7.0)
    cu = torch.tensor([2, 5, 5], dtype=torch.int32, device="cuda")
    contexts[dtype].cache_attention(c.c, q, o, cu=cu)
    assert bool((o[:2] == 7).all()) and bool((o[5:] == 7).all()) and bool((o[2:5] != 7).any())
    assert a.shape == o.shape


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,old,heads,kvh,window", [([70], [0], 3, 3, 0), ([200, 5], [100, 700], 8, 2, 0), ([130], [40], 2, 1, 33),
                                                      ([3], [2000], 64, 1, 0)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(contexts, dtype, dim, new, old, heads, kvh, window):
    """A value that is NaN or infinite, and a key that is NaN, in the middle of a chunk: rows
    before it (and those whose window has passed it) are as without it."""
    dt, g = TYPES[dtype], gen(13)
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], 16, kvh, dim)
    for s in range(len(new)):
        c.put(s, 0, old[s] + new[s], g)
    rows = sum(new)
    q, _ = rows_of((rows, heads, dim), dt, g)
    clean, o = torch.empty_like(q), torch.empty_like(q)
    cl, lse = torch.empty((rows, heads), device="cuda"), torch.empty((rows, heads), device="cuda")
    cu = offsets(new)
    contexts[dtype].cache_attention(c.c, q, clean, cu=cu, window=window, lse=cl)
    where = old[0] + new[0] // 2
    p, t = c.where(0, torch.tensor([where, where + 1], device="cuda"))
    c.v[p[0], t[0], 0, 5] = float("nan")
    c.v[p[1], t[1], kvh - 1, dim - 3] = float("-inf")
    contexts[dtype].cache_attention(c.c, q, o, cu=cu, window=window, lse=lse)
    assert torch.equal(lse, cl)                        # the weights do not know of values
    group = heads // kvh
    for r in range(rows):
        pos = old[0] + r if r < new[0] else -1
        for i, (hk, col) in enumerate([(0, 5), (kvh - 1, dim - 3)]):
            sees = pos >= where + i and (window == 0 or pos - (where + i) < window)
            got = o[r, hk * group:(hk + 1) * group, col]
            if sees:
                assert not bool(torch.isfinite(got).any()), (r, i)
                o[r, hk * group:(hk + 1) * group, col] = clean[r, hk * group:(hk + 1) * group, col]
    # everything else: sums in another order at most
    tol = 4 * HALF[dt] if dt == torch.bfloat16 else 64 * U
    assert bool(((o.double() - clean.double()).abs() <= tol * (1 + clean.double().abs())).all())
    # a key that is NaN
    c.k[p[0], t[0], 0, 2] = float("nan")
    c.v[p[0], t[0], 0, 5], c.v[p[1], t[1], kvh - 1, dim - 3] = 0.5, 0.5
    contexts[dtype].cache_attention(c.c, q, o, cu=cu, window=window, lse=lse)
    for r in range(new[0]):
        sees = old[0] + r >= where and (window == 0 or old[0] + r - where < window)
        assert bool(torch.isnan(o[r, :group]).all()) == sees, r
    assert bool(torch.isfinite(o[new[0]:]).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_one_sequence_without_offsets(contexts, dtype):
    dt, ctx, g = TYPES[dtype], contexts[dtype], gen(31)
    c = Paged(dt, [50], [120], 16, 4, 64)
    c.put(0, 0, 50, g)
    x = torch.randn((70, 3, 4, 64), device="cuda", generator=g).to(dt)
    ctx.cache_append(c.c, x[:, 1], x[:, 2])
    o, o2, lse = torch.empty_like(x[:, 0]), torch.empty_like(x[:, 0]), torch.empty((70, 4), device="cuda")
    ctx.cache_attention(c.c, x[:, 0], o, lse=lse)
    ctx.cache_attention(c.c, x[:, 0], o2, cu=offsets([70]))
    assert torch.equal(o, o2)
    check_cache_attention(c, x[:, 0], o, lse, [70], True, 0, 0.125, o, lse)
    ctx.cache_attention(c.c, x[:0, 0], o[:0])
    ctx.cache_append(c.c, x[:0, 1], x[:0, 2])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_pages_beyond_4_gb(contexts, dtype):
    """Pages whose byte offsets pass 32 bits, and a page that spans more by its heads' stride."""
    dt, g = TYPES[dtype], gen(35)
    es = 2 if dt == torch.bfloat16 else 4
    from paper_2609_38984_amd import swam
    ld = 1 << 20
    n = (5 << 30) // (ld * es) // 8 + 2
    buf = torch.zeros((n, 8, ld), dtype=dt, device="cuda")
    k, v = buf[:, :, :64].unflatten(2, (1, 64)), buf[:, :, -64:].unflatten(2, (1, 64))
    old, new = n * 8 - 60, 40
    pages = torch.randperm(n, device="cuda", generator=g)
    table = pages.to(torch.int32)[None]
    length = torch.tensor([0], dtype=torch.int32, device="cuda")
    cache = swam.Cache(k, v, table, length)
    x = torch.randn((old + new, 3, 1, 64), device="cuda", generator=g).to(dt)
    contexts[dtype].cache_append(cache, x[:old, 1], x[:old, 2])
    length.fill_(old)
    contexts[dtype].cache_append(cache, x[old:, 1], x[old:, 2])
    q = x[old:, 0].contiguous()
    o, lse = torch.empty_like(q), torch.empty((new, 1), device="cuda")
    contexts[dtype].cache_attention(cache, q, o, lse=lse)
    j = torch.arange(old + new, device="cuda")
    assert torch.equal(k[pages[j // 8], j % 8], x[:, 1]) and torch.equal(v[pages[j // 8], j % 8], x[:, 2])

    class C:
        kvh, lengths = 1, [old]
        where = staticmethod(lambda s, j: (pages[j // 8], j % 8))
    C.k, C.v = k, v
    check_cache_attention(C, q, o, lse, [new], True, 0, 0.125, o, lse)


# ---------------------------------------------------------------------------
# how they are called
# ---------------------------------------------------------------------------
def test_refusals_launch_nothing(contexts):
    from paper_2609_38984_amd import swam
    ctx, bf = contexts["bf16"], torch.bfloat16
    c = Paged(bf, [3, 3], [20, 20], 8, 2, 64, by_head=False, fill=5.0)
    x = torch.full((6, 3, 2, 64), 9.0, dtype=bf, device="cuda")
    q, k, v = x.unbind(1)
    cu, o = offsets([3, 3]), torch.full((6, 2, 64), 9.0, dtype=bf, device="cuda")
    post, _, _ = make_post(bf, 64, 64, True)
    for bad in (dict(k=k.float()), dict(v=v[:5]), dict(k=k[:, :1]), dict(cu=offsets([6])), dict(cu=cu.long()), dict(q=q[:4]),
                dict(q=q.cpu()), dict(q_out=o), dict(pos=torch.zeros(6, dtype=torch.int64, device="cuda")),
                dict(pos=torch.zeros(5, dtype=torch.int32, device="cuda")), dict(post=make_post(torch.float32, 64, 64, True)[0]),
                dict(post=make_post(bf, 128, 64, True)[0])):
        a = dict(k=k, v=v, cu=cu)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            ctx.cache_append(c.c, **a)
    for bad in (dict(q=q.float()), dict(o=o[:5]), dict(o=o[:, :, :32]), dict(cu=offsets([6])), dict(lse=torch.zeros(6, device="cuda")),
                dict(q=q[:, :, ::2])):
        a = dict(q=q, o=o, cu=cu)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            ctx.cache_attention(c.c, **a)
    for bad in (dict(q=q.float()), dict(k=k[:5]), dict(q=None, k=None), dict(q_out=o[:5]), dict(k=k[:, :, ::2])):
        a = dict(q=q, k=k)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            ctx.qk_norm_rope(post=post, **a)
    for bad in (lambda: swam.Cache(c.k, c.v[:1], c.table, c.length), lambda: swam.Cache(c.k, c.v.float(), c.table, c.length),
                lambda: swam.Cache(c.k, c.v, c.table.long(), c.length), lambda: swam.Cache(c.k, c.v, c.table, c.length[:1]),
                lambda: swam.Cache(c.k[..., ::2], c.v[..., ::2], c.table, c.length), lambda: swam.Cache(c.k.cpu(), c.v.cpu(), c.table, c.length),
                lambda: swam.Rope(freq_of(8).float()), lambda: swam.Rope(freq_of(8), "other"), lambda: swam.Rope(freq_of(8)[::2])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(swam.SwamError, match="overlaps"):
        ctx.cache_attention(c.c, o, o, cu=cu)
    with pytest.raises(swam.SwamError, match="overlaps"):
        ctx.cache_append(c.c, c.k[0, :6], v, cu=cu)
    with pytest.raises(swam.SwamError, match="SWAM_E_SHAPE"):
        ctx.qk_norm_rope(q, k, make_post(bf, 64, 66, True, gain=False)[0])
    with pytest.raises(swam.SwamError, match="window"):
        ctx.cache_attention(c.c, q, o, cu=cu, window=-1)
    torch.cuda.synchronize()
    assert bool((x == 9).all()) and bool((o == 9).all()) and bool((c.k == 5).all()) and bool((c.v == 5).all())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_results_repeat_and_do_not_depend_on_the_workspace(contexts, dtype):
    """Twice the same call gives the same bits; a context whose workspace holds few partial
    sums, or none, takes other splits within the same bounds."""
    from paper_2609_38984_amd import swam
    dt = TYPES[dtype]
    small = swam.Context(W.preset(1).replace(dtype=dtype, d_model=64, n_heads=1))
    for new, old, heads in (([1] * 3, [4000, 9, 700], 6), ([300], [2200], 4), ([40, 2], [60, 9000], 2)):
        o1 = run_cache_attention(contexts[dtype], dt, new, old, heads, heads, 64, 16, seed=43)
        o2 = run_cache_attention(contexts[dtype], dt, new, old, heads, heads, 64, 16, seed=43)
        assert torch.equal(o1, o2)
        run_cache_attention(small, dt, new, old, heads, heads, 64, 16, seed=43)


class Stream:
    """A policy's sequences in the middle of their episode: projections of chunk after chunk, appended
    and attended, the lengths moved on behind each."""

    def __init__(self, dt, chunks, page, heads, kvh, dim, seed, half):
        g = gen(seed)
        self.chunks, self.heads, self.kvh, self.dim = chunks, heads, kvh, dim
        total = [sum(c[s] for c in chunks) for s in range(len(chunks[0]))]
        self.c = Paged(dt, [0] * len(total), total, page, kvh, dim, seed)
        self.post, self.gains, self.freq = make_post(dt, dim, dim, half, seed=seed)
        self.half = half
        self.x = [torch.randn((sum(c), heads + 2 * kvh, dim), device="cuda", generator=g).to(dt) for c in chunks]
        self.cu = [offsets(c) for c in chunks]
        self.n = [torch.tensor(c, dtype=torch.int32, device="cuda") for c in chunks]
        self.q = [torch.empty((sum(c), heads, dim), dtype=dt, device="cuda") for c in chunks]
        self.o = [torch.empty((sum(c), heads, dim), dtype=dt, device="cuda") for c in chunks]

    def run(self, ctx, causal=True):
        self.c.length.zero_()
        for x, cu, n, q, o in zip(self.x, self.cu, self.n, self.q, self.o):
            qkv = x.split((self.heads, self.kvh, self.kvh), 1)
            ctx.cache_append(self.c.c, qkv[1], qkv[2], cu=cu, q=qkv[0], q_out=q, post=self.post)
            ctx.cache_attention(self.c.c, q, o, cu=cu, causal=causal)
            self.c.length.add_(n)
        return self.o


CHUNKS = [[40, 3, 0, 130], [1, 1, 1, 1], [70, 9, 500, 1], [1, 0, 1, 1], [17, 64, 1, 33]]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("heads,kvh,dim,page,half", [(4, 4, 64, 16, False), (6, 2, 128, 8, True), (3, 1, 64, 256, True)])
def test_a_stream_of_chunks(contexts, dtype, heads, kvh, dim, page, half):
    """Chunk after chunk through the cache gives what one causal pass over the whole sequences
    gives: in float64 from the projections, q and k rounded to storage where they are stored."""
    dt = TYPES[dtype]
    s = Stream(dt, CHUNKS, page, heads, kvh, dim, 5, half)
    s.run(contexts[dtype])
    start = [0] * 4
    for i, chunk in enumerate(CHUNKS):
        at = 0
        for b, n in enumerate(chunk):
            if n:
                j = torch.arange(start[b], start[b] + n, device="cuda")
                r = slice(at, at + n)
                check_close(s.q[i][r], *post64(s.x[i][r, :heads], j, True, 1e-6, s.gains[0], s.freq, half, 1.0), HALF[dt])
                p, t = s.c.where(b, j)
                check_close(s.c.k[p, t], *post64(s.x[i][r, heads:heads + kvh], j, True, 1e-6, s.gains[1], s.freq, half, 1.0), HALF[dt])
                assert torch.equal(s.c.v[p, t], s.x[i][r, heads + kvh:])
            at += n
        s.c.lengths = list(start)
        check_cache_attention(s.c, s.q[i], s.o[i], None, chunk, True, 0, dim ** -0.5, s.o[i], None)
        start = [a + n for a, n in zip(start, chunk)]
    assert s.c.length.tolist() == start


@pytest.mark.parametrize("dtype", list(TYPES))
def test_replayed_and_on_other_streams(contexts, dtype):
    """Two streams of chunks of one context, each captured once and replayed with eager work of the
    same context in between, give the eager bits every time, for new inputs in the same
    buffers too."""
    from paper_2609_38984_amd import swam
    dt = TYPES[dtype]
    stream = torch.cuda.Stream()
    ctx = swam.Context(W.preset(2).replace(dtype=dtype, n_blocks=1), stream)
    states = [Stream(dt, CHUNKS, 16, 4, 2, 64, 7, False), Stream(dt, [[900], [1], [1], [64]], 64, 4, 4, 128, 8, True)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for s in states:
            s.run(ctx)
    torch.cuda.synchronize()
    graphs = []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            s.run(ctx)
        graphs.append(g)
    for turn in range(4):
        for i, (s, g) in enumerate(zip(states, graphs)):
            for x in s.x:
                x.copy_(torch.randn(x.shape, device="cuda", generator=gen(70 + turn)).to(dt))
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                g.replay()
                kept = [t.clone() for t in s.o] + [s.c.k.clone(), s.c.v.clone()]
                for t in s.o:
                    t.zero_()
                s.run(ctx)
            torch.cuda.synchronize()
            for a, b in zip(kept, s.o + [s.c.k, s.c.v]):
                assert torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0)), (turn, i)
    other = torch.cuda.Stream()
    ctx.set_stream(other)
    with torch.cuda.stream(other):
        for t in states[0].o:
            t.zero_()
        want = [t.clone() for t in states[0].o]
        states[0].run(ctx)
    torch.cuda.synchronize()
    contexts[dtype].qk_norm_rope(states[0].q[0], None, states[0].post)
    assert any(bool((a != b).any()) for a, b in zip(want, states[0].o))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_two_contexts_at_once(contexts, dtype):
    """Two contexts on two streams, their calls in flight together, give what each gives alone."""
    from paper_2609_38984_amd import swam
    dt = TYPES[dtype]
    def made(i):
        return Stream(dt, CHUNKS if i == 0 else [[1500, 20], [1, 1], [1, 300]], 16, 4, 2, 64, 90 + i, bool(i))
    wants = []
    for i in range(2):
        s = made(i)
        wants.append([t.clone() for t in s.run(contexts[dtype])])
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [swam.Context(W.preset(2).replace(dtype=dtype, n_blocks=1), st) for st in streams]
    runs = [[made(i) for _ in range(4)] for i in range(2)]
    torch.cuda.synchronize()
    for n in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                runs[i][n].run(ctxs[i])
    torch.cuda.synchronize()
    for i in range(2):
        for r in runs[i]:
            for a, b in zip(wants[i], r.o):
                assert torch.equal(a, b)


def test_steps_and_cache_calls_share_a_context(contexts):
    """A step of the model between two chunks leaves both as they were (they use one workspace
    in turn), and the timers see the calls."""
    from helpers import dev, model_for
    from paper_2609_38984_amd import swam
    cfg = W.preset(2).replace(n_blocks=2)
    blocks, _, model = model_for(cfg)
    inp = W.make_inputs(cfg, blocks[0]["w_qkv"])
    ctx = swam.Context(cfg)
    x, temb = dev(inp.x(0), torch.bfloat16), dev(inp.temb(0))
    y = [torch.empty_like(x) for _ in range(2)]
    s = Stream(torch.bfloat16, [[700, 20], [1, 1]], 16, 4, 2, 64, 3, False)
    ctx.timer_enable(["HEAD_POST", "APPEND", "CACHE_ATTN"], 64)
    outs = []
    for i in range(2):
        outs.append([t.clone() for t in s.run(ctx)])
        ctx.step(model, x, temb, 0, y[i])
    ctx.qk_norm_rope(s.q[0], None, s.post)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert ctx.timer_read("HEAD_POST")[0] == 1 and ctx.timer_read("APPEND")[0] == 4 and ctx.timer_read("CACHE_ATTN")[0] == 4


# ---------------------------------------------------------------------------
# every form of the kernels
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("new,old", [([1, 1, 1], [700, 5, 2100]), ([20, 3], [333, 1500]), ([90, 200], [700, 61]), ([33], [0])])
def test_every_page_size(contexts, dtype, dim, page, new, old):
    """Loads of 8, 16, 32 and 64 keys to a page, for few rows and for chunks."""
    run_cache_attention(contexts[dtype], TYPES[dtype], new, old, 4, 2, dim, page, True, 0, page + dim)
    run_cache_attention(contexts[dtype], TYPES[dtype], new, old, 3, 3, dim, page, False, 150, page)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,old,heads,kvh,dim", [
    ([1500], [0], 56, 56, 64),                              # more row tiles than groups of waves take
    ([700, 300], [0, 900], 80, 80, 64),
    ([900], [300], 70, 70, 128),
    ([1300], [200], 24, 24, 64),                            # one sequence that fills the card unsplit
    ([1] * 40, [3000] + [40] * 38 + [1200], 16, 16, 64),     # cut lines of many rows
    ([2] * 30, [2500, 9] * 15, 32, 4, 128),
    ([1] * 100, [4000] + [(31 * i) % 300 for i in range(99)], 4, 2, 64),    # two sequences to a lane
    ([(13 * i) % 60 + 40 for i in range(80)], [3000] + [(17 * i) % 200 for i in range(79)], 2, 1, 64),
    ([1] * 300, [(41 * i) % 700 for i in range(300)], 2, 1, 128),
    ([1], [20000], 4, 1, 64), ([3, 1], [15000, 9], 8, 1, 128)])
def test_many_rows_long_lines_and_many_sequences(contexts, dtype, new, old, heads, kvh, dim):
    for causal, window in ((True, 0), (False, 0), (True, 700)):
        run_cache_attention(contexts[dtype], TYPES[dtype], new, old, heads, kvh, dim, 16, causal, window, heads + dim)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,old", [([1, 1], [5000, 300]), ([200], [3000]), ([30, 2], [900, 2000])])
def test_workspaces_of_any_size(dtype, new, old):
    """A context of one narrow block holds partial results of few slices, and one of a single
    short sequence of next to none; both give what the large one gives, within the bounds."""
    from paper_2609_38984_amd import swam
    for cfg in (W.preset(1).replace(dtype=dtype), W.preset(1).replace(dtype=dtype, d_model=64, n_heads=1),
                W.preset(1).replace(dtype=dtype, d_model=64, n_heads=1, n_ctx=0, n_frames=1, frame_h=2, frame_w=2, n_act=1, k_core=2,
                                    k_anchor=1)):
        ctx = swam.Context(cfg)
        for heads, kvh, dim in ((8, 2, 128), (6, 6, 64)):
            run_cache_attention(ctx, TYPES[dtype], new, old, heads, kvh, dim, 16, seed=3)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_strided_tables_shared_pages_and_repeated_sequences(contexts, dtype):
    """A table that is a column range of a wider one, a prompt whose pages several sequences
    share, and a page that stands in a table twice."""
    from paper_2609_38984_amd import swam
    dt, g = TYPES[dtype], gen(77)
    n, page, kvh = 12, 16, 2
    k, v = (torch.randn((n, page, kvh, 64), device="cuda", generator=g).to(dt) for _ in range(2))
    wide = torch.full((3, 9), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, 2:7] = torch.tensor([[0, 1, 2, 3, 4], [0, 1, 5, 5, 6], [0, 1, 7, 8, 9]], device="cuda")
    table = wide[:, 2:7]
    length = torch.tensor([70, 60, 33], dtype=torch.int32, device="cuda")
    cache = swam.Cache(k, v, table, length)
    new = [3, 1, 40]
    q, _ = rows_of((44, 4, 64), dt, g)
    o, lse = torch.empty_like(q), torch.empty((44, 4), device="cuda")
    contexts[dtype].cache_attention(cache, q, o, cu=offsets(new), lse=lse)

    class C:
        lengths = [70, 60, 33]
        where = staticmethod(lambda s, j: (table[s].long()[j // page], j % page))
    C.kvh, C.k, C.v = kvh, k, v
    check_cache_attention(C, q, o, lse, new, True, 0, 0.125, o, lse)


# ---------------------------------------------------------------------------
# what a sequence's neighbours do to it
# ---------------------------------------------------------------------------
FEW_ROWS = 32                                            # tokens times heads of a group


def check_fine(c, q, o, new, causal, window, scale):
    """Chunks of up to FEW_ROWS rows keep 16 bits of each weight, which stand as two bf16 numbers: the first is off
    by 2^-8 of it at most and the second by 2^-8 of that.  Else the bound of check_cache_attention."""
    heads, dim = q.shape[1:]
    group, h, at, checked = heads // c.kvh, HALF[q.dtype], 0, 0
    bits = 2.0 ** -16 if q.dtype == torch.bfloat16 else 0.0
    for s, n in enumerate(new):
        rows = slice(at, at + n)
        at += n
        if n == 0 or n * group > FEW_ROWS:
            continue
        total = c.lengths[s] + n
        j = torch.arange(total, device="cuda")
        i = torch.arange(c.lengths[s], total, device="cuda")[:, None]
        see = torch.ones((n, total), dtype=torch.bool, device="cuda")
        if causal:
            see &= j <= i
        if window:
            see &= i - j < window
        p, t = c.where(s, j)
        k, v = c.k[p, t].double(), c.v[p, t].double()
        for hd in range(heads):
            kj, vj, qj = k[:, hd // group], v[:, hd // group], q[rows, hd].double()
            x = (qj @ kj.t().contiguous() * scale).masked_fill(~see, -math.inf)
            lse = torch.logsumexp(x, 1, keepdim=True)
            w = torch.exp(x - lse)
            want, size = w @ vj, w @ vj.abs()
            qk = ((qj.abs() @ kj.abs().t().contiguous()) * scale).masked_fill(~see, 0.0).amax(1, keepdim=True)
            lerr, sums = 2 * (dim + 8) * U * qk + 8 * U * lse.abs(), (total + 16) * U
            err = (bits + 2 * lerr + 2 * sums) * 1.01 * size
            err = err + (h + 4 * U) * (want.abs() + err)
            off = (o[rows, hd].double() - want).abs()
            assert bool((off <= err).all()), (s, hd, float((off / err).max()))
            checked += off.numel()
    assert checked


def run_fine(ctx, dt, new, old, heads, kvh, dim, page, causal=True, window=0, seed=0):
    """Even weights: the logits' own errors, which the bound grows with, are small beside the weights'."""
    g = gen(seed)
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], page, kvh, dim, seed)
    for s in range(len(new)):
        c.put(s, 0, old[s] + new[s], g)
    q, _ = rows_of((sum(new), heads, dim), dt, g)
    o = torch.empty_like(q)
    ctx.cache_attention(c.c, q, o, cu=offsets(new), causal=causal, window=window, scale=0.01)
    check_fine(c, q, o, new, causal, window, 0.01)
    check_cache_attention(c, q, o, None, new, causal, window, 0.01, o, None)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,old,heads,kvh,dim,page", [
    ([1248, 1, 1, 7], [500, 3000, 40, 90], 4, 2, 64, 64), ([3, 400, 1], [70, 0, 200], 3, 3, 64, 8), ([300, 5, 1], [60, 77, 1000], 12, 3, 128, 16),
    ([1, 200, 2, 0, 8], [128, 100, 31, 9, 63], 4, 1, 128, 32), ([1, 700, 16], [90, 64, 64], 160, 80, 64, 16),
    ([500, 1, 4], [0, 55, 800], 70, 70, 128, 64)])
def test_short_chunks_beside_long_ones_keep_16_bits_of_the_weights(contexts, dtype, new, old, heads, kvh, dim, page):
    for causal, window in ((True, 0), (False, 0), (True, 50), (False, 33)):
        run_fine(contexts[dtype], TYPES[dtype], new, old, heads, kvh, dim, page, causal, window, 11)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,old,heads,kvh,dim,page", [
    ([1] * 8, [60 * i for i in range(8)], 4, 4, 64, 32), ([1], [3000], 14, 2, 128, 64), ([3, 8, 1], [200, 64, 5], 8, 2, 64, 8),
    ([1] * 70, [(37 * i) % 400 for i in range(70)], 6, 3, 128, 16), ([32], [100], 2, 2, 64, 16), ([8], [900], 12, 3, 128, 256)])
def test_single_tokens_and_short_chunks_keep_16_bits_of_the_weights(contexts, dtype, new, old, heads, kvh, dim, page):
    for causal, window in ((True, 0), (False, 0), (True, 50)):
        run_fine(contexts[dtype], TYPES[dtype], new, old, heads, kvh, dim, page, causal, window, 12)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,old,heads,kvh", [
    ([1], [900], 4, 2), ([1, 1, 1], [40, 500, 2000], 3, 3), ([3], [2000], 8, 1), ([200], [300], 4, 4), ([300, 1, 4], [64, 700, 90], 4, 2),
    ([1] * 70, [100 + 3 * i for i in range(70)], 4, 4)])
def test_infinite_values_stay_infinite(contexts, dtype, dim, new, old, heads, kvh):
    """A value that is infinite, with a weight above zero, makes its sign's infinity of its column in the rows that
    see it, not NaN, in whichever way the weights are held; the others stay finite."""
    dt, g = TYPES[dtype], gen(17)
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], 16, kvh, dim)
    q, _ = rows_of((sum(new), heads, dim), dt, g)
    hit = []
    for s in range(len(new)):
        c.put(s, 0, old[s] + new[s], g)
        # of a key that all rows see, and one that a chunk's first rows do not
        for j, head, col, value in ((old[s] // 2, 0, 3, math.inf), (old[s] + new[s] // 2, kvh - 1, dim - 6, -math.inf)):
            p, t = c.where(s, torch.tensor([j], device="cuda"))
            c.v[p[0], t[0], head, col] = value
            hit.append((s, j, head, col, value))
    for causal in (True, False):
        o = torch.empty_like(q)
        contexts[dtype].cache_attention(c.c, q, o, cu=offsets(new), causal=causal, scale=0.01)
        want = torch.zeros((sum(new), heads, dim), device="cuda")
        group, start = heads // kvh, offsets(new).tolist()
        for s, j, head, col, value in hit:
            i = torch.arange(new[s], device="cuda")
            sees = (old[s] + i >= j) | (not causal)
            want[start[s]:start[s + 1], head * group:(head + 1) * group, col] = torch.where(sees, value, 0.0)[:, None]
        odd = torch.isinf(want)
        assert torch.equal(o.float()[odd], want[odd])
        assert bool(torch.isfinite(o[~odd]).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("new,old,heads,kvh,dim", [
    ([1248] + [1] * 63, [100] + [(61 * i) % 900 for i in range(63)], 3, 3, 64),      # by their mean, single tokens
    ([1] * 40 + [700] + [1] * 23, [30] * 64, 4, 2, 128), ([0] * 100 + [900] + [0] * 155, [0] * 100 + [500] + [9] * 155, 4, 4, 64),
    ([600] + [0] * 1023, [0] * 1024, 6, 3, 64), ([0, 0, 33, 0, 0, 0, 1, 0], [70, 0, 900, 3, 0, 0, 64, 1], 2, 1, 64)])
def test_a_long_chunk_among_single_tokens_and_idle_sequences(contexts, dtype, new, old, heads, kvh, dim):
    for causal, window in ((True, 0), (False, 0), (True, 130)):
        run_cache_attention(contexts[dtype], TYPES[dtype], new, old, heads, kvh, dim, 16, causal, window, 19)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cu,rows", [
    ([-9, 20, 20, 60, 1 << 30], 80),                      # below the rows, an empty one, past the rows
    ([30, 10, 40, 55], 60),                               # falling: the first is empty, rows 0 to 9 and 55 on are nobody's
    ([5, 5, -3, -7, 12, 31], 40), ([1 << 30, 9, 22], 22), ([7, -(1 << 31), (1 << 31) - 1], 19),
    ([50] + [3] * 70 + [3 + i // 3 for i in range(100)], 36), ([10] * 60 + [0, 10, 12, 36] + [36] * 40, 38),
    ([30, 40, 20, 30, 0, 20], 43)])                       # not in the order of their rows
def test_append_and_attention_within_clamped_and_falling_offsets(contexts, dtype, cu, rows):
    """Sequence s is the rows from cu[s] to cu[s + 1], both clamped to the rows, and empty where they fall.  What is
    appended, what it is attended with, and what is nobody's and left as it was."""
    dt, g = TYPES[dtype], gen(23)
    seqs = len(cu) - 1
    ends = [min(max(e, 0), rows) for e in cu[1:]]
    starts = [min(max(b, 0), e) for b, e in zip(cu, ends)]
    new = [e - b for b, e in zip(starts, ends)]
    old = [(11 * s) % 40 + 900 * (s % 5 == 3) for s in range(seqs)]     # (keys of the longer ones are split)
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], 8, 2, 64, fill=5.0)
    for s in range(seqs):
        c.put(s, 0, old[s], g)
    q, k, v = (torch.randn((rows, n, 64), device="cuda", generator=g).to(dt) for n in (4, 2, 2))
    want_k, want_v, mine = c.k.clone(), c.v.clone(), torch.zeros(rows, dtype=torch.bool, device="cuda")
    for s in range(seqs):
        if new[s]:
            p, t = c.where(s, torch.arange(old[s], old[s] + new[s], device="cuda"))
            want_k[p, t], want_v[p, t] = k[starts[s]:ends[s]], v[starts[s]:ends[s]]
            assert not bool(mine[starts[s]:ends[s]].any())        # no row is two sequences'
            mine[starts[s]:ends[s]] = True
    at = torch.tensor(cu, device="cuda").to(torch.int32)
    qo = torch.full_like(q, 9.0)
    contexts[dtype].cache_append(c.c, k, v, cu=at, q=q, q_out=qo)
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v)
    assert torch.equal(qo[mine], q[mine]) and bool((qo[~mine] == 9.0).all())
    o, lse = torch.full_like(q, 7.0), torch.full((rows, 4), 7.0, device="cuda")
    contexts[dtype].cache_attention(c.c, q, o, cu=at, lse=lse)
    assert bool((o[~mine] == 7.0).all()) and bool((lse[~mine] == 7.0).all())
    for s in range(seqs):
        if new[s]:
            r = slice(starts[s], ends[s])

            class One:
                kvh, k, v, lengths = c.kvh, c.k, c.v, [old[s]]
                where = staticmethod(lambda _, j, s=s: c.where(s, j))
            check_cache_attention(One, q[r], o[r], lse[r], [new[s]], True, 0, 0.125, o[r], lse[r])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_context_that_moves_to_another_stream_gives_the_same(dtype):
    """The same calls behind set_stream give the bits of those in front of it."""
    from paper_2609_38984_amd import swam
    dt = TYPES[dtype]
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = swam.Context(W.preset(2).replace(dtype=dtype, n_blocks=1), first)
    s = Stream(dt, CHUNKS, 16, 4, 2, 64, 7, False)
    torch.cuda.synchronize()
    kept = []
    for stream in (first, second, first):
        ctx.set_stream(stream)
        with torch.cuda.stream(stream):
            for t in s.o + s.q + [s.c.k, s.c.v]:
                t.zero_()
            s.run(ctx)
            turned = torch.empty_like(s.q[0])
            ctx.qk_norm_rope(s.q[0], None, s.post, q_out=turned)
            kept.append([t.clone() for t in s.o + s.q + [s.c.k, s.c.v, turned]])
        torch.cuda.synchronize()
    assert all(bool((t != 0).any()) for t in kept[0])
    for other in kept[1:]:
        for a, b in zip(kept[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,old,rows,heads,kvh,dim,page", [
    (1, 70, 200, 4, 4, 64, 16), (8, 200, 1000, 8, 2, 64, 64), (20, 33, 700, 3, 3, 128, 8), (3, 900, 2000, 100, 50, 64, 32)])
def test_a_short_chunk_in_a_padded_call_keeps_16_bits_of_the_weights(contexts, dtype, n, old, rows, heads, kvh, dim, page):
    """One sequence whose offsets leave most rows out, as a captured call of the longest chunk has them."""
    dt, g = TYPES[dtype], gen(29)
    c = Paged(dt, [old], [old + n], page, kvh, dim)
    c.put(0, 0, old + n, g)
    for first in (0, rows - n, 40):
        q, _ = rows_of((rows, heads, dim), dt, g)
        o = torch.full_like(q, 7.0)
        cu = torch.tensor([first, first + n], dtype=torch.int32, device="cuda")
        contexts[dtype].cache_attention(c.c, q, o, cu=cu, scale=0.01)
        r = slice(first, first + n)
        check_fine(c, q[r], o[r], [n], True, 0, 0.01)
        check_cache_attention(c, q[r], o[r], None, [n], True, 0, 0.01, o[r], None)
        assert bool((o[:first] == 7.0).all()) and bool((o[first + n:] == 7.0).all())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,old,heads,kvh", [([1], [9], 4, 2), ([1], [3000], 4, 4), ([5, 1], [40, 900], 6, 2), ([200], [150], 3, 3),
                                               ([300, 2], [64, 700], 4, 4), ([900], [0], 16, 16)])
def test_rows_without_a_weight_are_zeros_whatever_the_values(contexts, dtype, dim, new, old, heads, kvh):
    """Scores that are all minus infinity: the rows are zeros and their normaliser minus infinity, also with values that are
    not finite, in a cache whose first K/V head alone is so."""
    dt, g = TYPES[dtype], gen(31)
    c = Paged(dt, old, [a + b for a, b in zip(new, old)], 16, kvh, dim)
    for s in range(len(new)):
        c.put(s, 0, old[s] + new[s], g)
    q, _ = rows_of((sum(new), heads, dim), dt, g)
    q[:, :, 7] = q[:, :, 7].abs() + 0.5
    clean = torch.empty_like(q)
    contexts[dtype].cache_attention(c.c, q, clean, cu=offsets(new))
    for s in range(len(new)):
        j = torch.arange(old[s] + new[s], device="cuda")
        p, t = c.where(s, j)
        c.k[p, t, 0, 7] = -math.inf
        c.v[p, t, 0] = torch.tensor([math.inf, math.nan, -math.inf, 1.0], device="cuda").to(dt)[(j[:, None] + torch.arange(dim, device="cuda")) % 4]
    o, lse = torch.full_like(q, 7.0), torch.full((sum(new), heads), 7.0, device="cuda")
    contexts[dtype].cache_attention(c.c, q, o, cu=offsets(new), lse=lse)
    group = heads // kvh
    assert bool((o[:, :group] == 0).all()) and bool((lse[:, :group] == -math.inf).all())
    assert torch.equal(o[:, group:], clean[:, group:]) and bool(torch.isfinite(lse[:, group:]).all())
