"""Host-side checks of the operators of swam_cache.h (no GPU): exports, the frequencies of
the rotation, and every refusal.  A call is checked before its context, so a NULL
context shows what is wrong with the call itself; fake pointers are never dereferenced."""
import ctypes as C
import math
import os
import random
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE = -1, -2


@pytest.fixture(scope="module")
def lib():
    from paper_2609_38984_amd import swam
    if not os.path.exists(swam.LIB_PATH):
        from paper_2609_38984_amd.build import build
        build()
    return swam.load_library()


def test_every_declared_operator_is_exported(lib):
    from paper_2609_38984_amd import swam
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "swam_cache.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(swam_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(swam.CACHE_EXPORTS)
    for n in names:
        assert hasattr(lib, n), n
    for name, value in re.findall(r"#define SWAM_(CACHE_MAX_SEQS|CACHE_MAX_PAGE|QK_MAX_DIM)\s+(\d+)", text):
        assert getattr(swam, name) == int(value)
    for names, prefix in ((swam.ROPE_LAYOUTS, "ROPE_"), (swam.ROPE_SCALINGS, "ROPE_")):
        for name, value in names.items():
            assert f"SWAM_{prefix}{name.upper()} = {value}" in text
    # the classes of the timers stand in the header's order
    head = open(os.path.join(ROOT, "include", "swam.h")).read()
    listed = re.findall(r"SWAM_T_([A-Z0-9_]+)", head[head.index("SWAM_T_ADALN = 0"):head.index("SWAM_T_COUNT\n")])
    assert listed[:len(swam.TIMERS)] == swam.TIMERS


# ---------------------------------------------------------------------------
# frequencies
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dims", [2, 10, 64, 128, 512])
def test_frequencies(lib, dims):
    from paper_2609_38984_amd import swam
    theta = [10000.0 ** (-2.0 * i / dims) for i in range(dims // 2)]

    def same(a, b):
        assert len(a) == len(b) and all(abs(x - y) <= 1e-14 * y for x, y in zip(a, b))

    same(swam.rope_frequencies(dims)[0], theta)
    f, m = swam.rope_frequencies(dims, scaling="linear", factor=4.0)
    same(f, [t / 4.0 for t in theta])
    assert m == 1.0
    if dims > 2:
        f, m = swam.rope_frequencies(dims, scaling="ntk", factor=8.0)
        # the first pair keeps its frequency, the last is slowed by the whole factor
        assert m == 1.0 and f[0] == 1.0 and abs(f[-1] * 8.0 / theta[-1] - 1.0) < 1e-12
    f, m = swam.rope_frequencies(dims, scaling="yarn", factor=8.0, trained=4096.0)
    assert m == pytest.approx(0.1 * math.log(8.0) + 1.0, rel=2.0 ** -23)
    for x, t in zip(f, theta):
        turns = 4096.0 * t / (2.0 * math.pi)
        if turns >= 32.0:
            assert x == pytest.approx(t, rel=1e-14)
        elif turns <= 1.0:
            assert x == pytest.approx(t / 8.0, rel=1e-14)
        else:
            assert t / 8.0 < x < t
    # a factor of one changes nothing
    for scaling in swam.ROPE_SCALINGS:
        if dims > 2 or scaling != "ntk":
            f, m = swam.rope_frequencies(dims, scaling=scaling, trained=100.0)
            same(f, theta)
            assert m == 1.0


@pytest.mark.parametrize("kw", [
    dict(dims=0), dict(dims=3), dict(dims=514), dict(dims=-2), dict(dims=8, base=1.0), dict(dims=8, base=float("nan")),
    dict(dims=8, base=float("inf")), dict(dims=8, factor=0.5), dict(dims=8, factor=float("inf")),
    dict(dims=2, scaling="ntk", factor=2.0), dict(dims=8, scaling="yarn", factor=2.0),
    dict(dims=8, scaling="yarn", factor=2.0, trained=float("nan"))])
def test_frequencies_refuse(lib, kw):
    from paper_2609_38984_amd import swam
    with pytest.raises(swam.SwamError):
        swam.rope_frequencies(**kw)
    with pytest.raises(ValueError):
        swam.rope_frequencies(8, scaling="other")
    out = (C.c_double * 4)()
    assert lib.swam_rope_frequencies(8, 1e4, 0, 1.0, 0.0, None, C.byref(C.c_float())) == INVALID
    assert lib.swam_rope_frequencies(8, 1e4, 0, 1.0, 0.0, out, None) == INVALID
    assert lib.swam_rope_frequencies(8, 1e4, 4, 1.0, 0.0, out, C.byref(C.c_float())) == INVALID


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def _p(i):
    """A pointer of its own 64 GB range, 256-byte aligned."""
    return (i + 1) << 36


POST = dict(norm=1, eps=1e-6, q_gain=_p(20), k_gain=_p(21), rope_dims=32, rope_layout=1, rope_freq=_p(22),
            rope_magnitude=1.0)
CACHE = dict(k=_p(10), v=_p(11), k_page=64 * 2 * 16, k_token=64, k_head=64 * 16, v_page=64 * 2 * 16, v_token=64,
             v_head=64 * 16, n_pages=20, page_size=16, n_kv_heads=2, head_dim=64, n_seqs=3, max_pages=8,
             table_stride=8, table=_p(12), length=_p(13))
HEADS = dict(post=POST, pos=_p(0), q=_p(1), qs=256, k=_p(2), ks=128, rows=10, heads=4, kv=2, dim=64, qo=_p(3), qos=256,
             ko=_p(4), kos=128)
APPEND = dict(cache=CACHE, post=POST, pos=_p(0), cu=_p(1), q=_p(2), qs=256, k=_p(3), ks=128, v=_p(4), vs=128, rows=10,
              heads=4, qo=_p(5), qos=256)
ATTN = dict(cache=CACHE, cu=_p(1), q=_p(2), qs=256, rows=10, heads=4, causal=1, window=0, scale=0.125, o=_p(5), os=256,
            lse=_p(6))
CALLS = {"swam_qk_norm_rope": HEADS, "swam_cache_append": APPEND, "swam_cache_attention": ATTN}


def _call(lib, fn, change):
    """The call with some arguments changed; "cache.x" and "post.x" change the descriptors."""
    from paper_2609_38984_amd import swam
    a, kinds = dict(CALLS[fn]), {"cache": swam.CacheStruct, "post": swam.QkPostStruct}
    for n in kinds:
        if a.get(n) is not None:
            a[n] = dict(a[n])
    for n, v in change.items():
        if "." in n:
            a[n.split(".")[0]][n.split(".")[1]] = v
        else:
            a[n] = v
    for n, kind in kinds.items():
        if a.get(n) is not None:
            a[n] = C.byref(kind(**a[n]))
    rc = getattr(lib, fn)(None, *a.values())
    return rc, lib.swam_last_error(None).decode()


GOOD = {
    "swam_qk_norm_rope": [
        {}, dict(qo=_p(1)), dict(ko=_p(2)), dict(pos=None), dict(q=None, qo=None, heads=0),
        dict(k=None, ko=None, kv=0), dict(rows=0, q=None, k=None, qo=None, ko=None),
        {"post.norm": 0, "post.q_gain": None, "post.k_gain": None}, {"post.rope_dims": 0, "post.rope_freq": None},
        {"post.rope_dims": 64}, {"post.rope_dims": 2}, {"post.eps": 0.0},
        dict(dim=512, qs=2048, ks=1024, qos=2048, kos=1024), {"dim": 8, "post.rope_dims": 8},
        dict(qs=512, ks=512, k=_p(1) + 512, qos=512, kos=512, qo=_p(3), ko=_p(3) + 512)],   # column ranges of one buffer
    "swam_cache_append": [
        {}, dict(post=None), dict(pos=None), dict(q=None, qo=None, heads=0), dict(qo=_p(2)), dict(rows=0),
        {"cu": None, "cache.n_seqs": 1}, {"cache.n_pages": 0, "cache.k": None, "cache.v": None},
        {"cache.max_pages": 0, "cache.table": None},
        # tokens first, heads inside; K and V of a page side by side
        {"cache.k_token": 128, "cache.k_head": 64}, {"cache.v": _p(10) + 64 * 2 * 16 * 2, "cache.k_page": 4096, "cache.v_page": 4096},
        {"cache.n_seqs": 1024}, {"cache.page_size": 4096, "cache.k_head": 1 << 18, "cache.v_head": 1 << 18,
                                 "cache.k_page": 1 << 19, "cache.v_page": 1 << 19}],
    "swam_cache_attention": [
        {}, dict(causal=0), dict(window=1), dict(window=(1 << 31) - 1), dict(lse=None), dict(rows=0, q=None, o=None),
        dict(heads=2, qs=128, os=128), dict(qs=512, os=512, o=_p(2) + 512), {"cu": None, "cache.n_seqs": 1}],
}


@pytest.mark.parametrize("fn", list(CALLS))
def test_good_calls_only_lack_their_context(lib, fn):
    for change in GOOD[fn]:
        assert _call(lib, fn, change) == (INVALID, "ctx is NULL"), change


@pytest.mark.parametrize("change,code,word", [
    ({"post.norm": 2}, INVALID, "norm"), ({"post.eps": -1.0}, INVALID, "eps"), ({"post.eps": float("nan")}, INVALID, "eps"),
    ({"post.norm": 0}, INVALID, "gain"), ({"post.q_gain": _p(20) + 2}, INVALID, "16-byte"),
    ({"post.k_gain": _p(21) + 8}, INVALID, "16-byte"), ({"post.rope_dims": 3}, SHAPE, "rope_dims"),
    ({"post.rope_dims": 66}, SHAPE, "rope_dims"), ({"post.rope_dims": -2}, SHAPE, "rope_dims"),
    ({"post.rope_layout": 2}, INVALID, "rope_layout"), ({"post.rope_freq": None}, INVALID, "rope_freq"),
    ({"post.rope_freq": _p(22) + 4}, INVALID, "element type"), ({"post.rope_magnitude": float("inf")}, INVALID, "magnitude"),
    (dict(pos=_p(0) + 2), INVALID, "element type"), (dict(rows=-1), INVALID, "rows"), (dict(rows=1 << 31), SHAPE, "rows"),
    (dict(q=None), INVALID, "q required"), (dict(k=None), INVALID, "k required"), (dict(qo=None), INVALID, "q_out required"),
    (dict(qs=248), INVALID, "stride"), (dict(ks=64), INVALID, "stride"), (dict(qos=0), INVALID, "stride"),
    (dict(qs=1 << 46), SHAPE, "2^48"), (dict(q=_p(1) + 8), INVALID, "16-byte"), (dict(ks=132), INVALID, "16-byte"),
    (dict(heads=-1), INVALID, "heads"), (dict(heads=0, qo=None), INVALID, "without heads"),
])
def test_head_rows_are_refused(lib, change, code, word):
    for fn in ("swam_qk_norm_rope", "swam_cache_append"):
        rc, msg = _call(lib, fn, change)
        assert rc == code and word in msg, (fn, msg)


@pytest.mark.parametrize("change,code,word", [
    (dict(post=None), INVALID, "post"), (dict(dim=0), SHAPE, "head_dim"), (dict(dim=60), SHAPE, "head_dim"),
    (dict(dim=520, qs=4096, ks=4096, qos=4096, kos=4096), SHAPE, "head_dim"), (dict(kv=-1), INVALID, "heads"),
    (dict(heads=65535), SHAPE, "2^16"), (dict(ko=None), INVALID, "k_out required"), (dict(kos=120), INVALID, "stride"),
    (dict(ko=_p(4) + 2), INVALID, "16-byte"), (dict(qo=_p(1) + 512), INVALID, "overlaps"),
    (dict(qo=_p(1), qos=512), INVALID, "overlaps"), (dict(qo=_p(2)), INVALID, "overlaps"), (dict(ko=_p(1)), INVALID, "overlaps"),
    (dict(ko=_p(3) + 256), INVALID, "overlaps"), (dict(qo=_p(0) - 256), INVALID, "overlaps an input"),
    (dict(ko=_p(20)), INVALID, "overlaps an input"), (dict(qo=_p(21) - 1024), INVALID, "overlaps an input"),
    (dict(qo=_p(22)), INVALID, "overlaps an input"),
])
def test_qk_norm_rope_refuses(lib, change, code, word):
    rc, msg = _call(lib, "swam_qk_norm_rope", change)
    assert rc == code and word in msg, msg


@pytest.mark.parametrize("change,code,word", [
    (dict(cache=None), INVALID, "cache"), ({"cache.head_dim": 80}, SHAPE, "head_dim"), ({"cache.n_kv_heads": 0}, SHAPE, "heads"),
    ({"cache.n_kv_heads": 1 << 16}, SHAPE, "heads"), ({"cache.page_size": 4}, SHAPE, "page_size"),
    ({"cache.page_size": 24}, SHAPE, "page_size"), ({"cache.page_size": 8192}, SHAPE, "page_size"),
    ({"cache.n_seqs": 0}, SHAPE, "sequences"), ({"cache.n_seqs": 1025}, SHAPE, "sequences"),
    ({"cache.n_pages": -1}, INVALID, "n_pages"), ({"cache.max_pages": -1}, INVALID, "n_pages"),
    ({"cache.max_pages": 1 << 26, "cache.table_stride": 1 << 26}, SHAPE, "2^30"), (dict(cu=None), INVALID, "cu"),
    ({"cache.table": None}, INVALID, "table"), ({"cache.length": None}, INVALID, "length"),
    ({"cache.table_stride": 7}, INVALID, "table_stride"), ({"cache.table_stride": 1 << 47}, SHAPE, "2^48"),
    ({"cache.table": _p(12) + 2}, INVALID, "element type"), ({"cache.length": _p(13) + 1}, INVALID, "element type"),
    (dict(cu=_p(1) + 2), INVALID, "element type"), ({"cache.k": None}, INVALID, "required"), ({"cache.v": None}, INVALID, "required"),
    ({"cache.k_token": 56}, INVALID, "meet"), ({"cache.k_head": 512}, INVALID, "meet"), ({"cache.v_page": 1024}, INVALID, "meet"),
    ({"cache.k_page": 0}, INVALID, "meet"), ({"cache.k_page": -2048}, INVALID, "meet"), ({"cache.k_page": 1 << 46}, SHAPE, "2^48"),
    ({"cache.k_token": 1 << 22, "cache.k_head": 64, "cache.k_page": 1 << 27}, SHAPE, "2^22"),
    ({"cache.k": _p(10) + 8}, INVALID, "16-byte"), ({"cache.k_page": 2052}, INVALID, "16-byte"),
    ({"cache.v_head": 1028, "cache.v_page": 4096}, INVALID, "16-byte"), ({"cache.v": _p(10)}, INVALID, "one tensor"),
])
def test_caches_are_refused(lib, change, code, word):
    for fn in ("swam_cache_append", "swam_cache_attention"):
        rc, msg = _call(lib, fn, change)
        assert rc == code and word in msg, (fn, msg)


@pytest.mark.parametrize("change,code,word", [
    (dict(v=None), INVALID, "v required"), (dict(vs=64), INVALID, "stride"), (dict(v=_p(4) + 2), INVALID, "16-byte"),
    (dict(heads=65532, qs=1 << 23, qos=1 << 23), SHAPE, "2^16"), (dict(qo=_p(2) + 512), INVALID, "overlaps q"),
    (dict(qo=_p(3)), INVALID, "overlaps an input"), (dict(qo=_p(4)), INVALID, "overlaps an input"), (dict(qo=_p(1)), INVALID, "overlaps an input"),
    (dict(qo=_p(12)), INVALID, "overlaps an input"), (dict(qo=_p(13)), INVALID, "overlaps an input"),
    (dict(qo=_p(20)), INVALID, "overlaps an input"), (dict(k=_p(10)), INVALID, "cache overlaps"),
    (dict(v=_p(11) + 20 * 4096 - 256), INVALID, "cache overlaps"), (dict(q=_p(10) + 4096), INVALID, "cache overlaps"),
    (dict(qo=_p(11)), INVALID, "cache overlaps"), ({"cache.length": _p(10) + 64}, INVALID, "cache overlaps"),
    ({"cache.table": _p(11) - 16}, INVALID, "cache overlaps"),
])
def test_append_refuses(lib, change, code, word):
    rc, msg = _call(lib, "swam_cache_append", change)
    assert rc == code and word in msg, msg


@pytest.mark.parametrize("change,code,word", [
    (dict(heads=0), INVALID, "n_heads"), (dict(heads=5), INVALID, "n_heads"), (dict(heads=4098, qs=1 << 19, os=1 << 19), SHAPE, "4096"),
    (dict(rows=-1), INVALID, "rows"), (dict(rows=1 << 28), SHAPE, "2^30"), (dict(rows=1 << 62), SHAPE, "2^30"),
    (dict(causal=2), INVALID, "causal"), (dict(window=-1), INVALID, "window"),
    (dict(scale=0.0), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(q=None), INVALID, "q required"), (dict(o=None), INVALID, "o required"), (dict(qs=255), INVALID, "stride"),
    (dict(os=128), INVALID, "stride"), (dict(qs=1 << 22), SHAPE, "2^22"), (dict(q=_p(2) + 8), INVALID, "16-byte"),
    (dict(os=260), INVALID, "16-byte"), (dict(lse=_p(6) + 1), INVALID, "element type"),
    (dict(o=_p(2) + 512), INVALID, "overlaps an input"), (dict(o=_p(10) + 64), INVALID, "overlaps an input"),
    (dict(lse=_p(12)), INVALID, "overlaps an input"), (dict(lse=_p(5) + 512), INVALID, "o overlaps lse"),
])
def test_attention_refuses(lib, change, code, word):
    rc, msg = _call(lib, "swam_cache_attention", change)
    assert rc == code and word in msg, msg


def _joint(shift, **change):
    """K and V in one buffer, V `shift` bytes behind K."""
    a = {"cache.v": _p(10) + shift}
    a.update({"cache." + n: v for n, v in change.items()})
    return a


# elements of a head, a token's heads, a head's tokens and a page of CACHE (head by head)
HEAD, PAGE = 64, 64 * 2 * 16


@pytest.mark.parametrize("change", [
    # one token, one head or one page apart, to either side, and by less than a head
    _joint(2 * HEAD), _joint(-2 * HEAD), _joint(2 * HEAD * 16), _joint(-2 * HEAD * 16), _joint(2 * PAGE), _joint(-2 * PAGE),
    _joint(16), _joint(-16), _joint(2 * (19 * PAGE + HEAD * 16 + 15 * HEAD)), _joint(2 * 20 * PAGE - 16),
    # tokens of both heads in turn
    _joint(2 * HEAD, k_token=128, v_token=128, k_head=64, v_head=64), _joint(256, k_token=128, v_token=128, k_head=64, v_head=64),
    # a page of both, V one token or one page too early or too late
    _joint(2 * PAGE - 2 * HEAD, k_page=2 * PAGE, v_page=2 * PAGE), _joint(2 * PAGE + 2 * HEAD, k_page=2 * PAGE, v_page=2 * PAGE),
    _joint(4 * PAGE, k_page=2 * PAGE, v_page=2 * PAGE),
    # other strides inside or between the pages
    _joint(2 * HEAD, k_page=2 * PAGE, v_page=4 * PAGE), _joint(2 * HEAD * 16, v_token=128, v_head=64),
    _joint(2 * PAGE - 256, k_page=2 * PAGE, v_page=2 * PAGE, v_token=128, v_head=64),
])
def test_keys_and_values_that_overlap_are_refused(lib, change):
    for fn in ("swam_cache_append", "swam_cache_attention"):
        rc, msg = _call(lib, fn, change)
        assert rc == INVALID and "k and v overlap" in msg, (fn, msg)


@pytest.mark.parametrize("change", [
    # behind each other
    _joint(2 * 20 * PAGE), _joint(-2 * 20 * PAGE), _joint(2 * 20 * PAGE, v_token=128, v_head=64),
    # K and V of a page side by side, in either order, laid out alike or not
    _joint(2 * PAGE, k_page=2 * PAGE, v_page=2 * PAGE), _joint(-2 * PAGE, k_page=2 * PAGE, v_page=2 * PAGE),
    _joint(2 * PAGE, k_page=2 * PAGE, v_page=2 * PAGE, v_token=128, v_head=64),
    # of a token (all heads of K, then of V), of a head's tokens, of a token and head
    _joint(2 * 128, k_token=256, v_token=256, k_head=64, v_head=64, k_page=2 * PAGE, v_page=2 * PAGE),
    _joint(2 * HEAD * 16, k_head=2 * HEAD * 16, v_head=2 * HEAD * 16, k_page=2 * PAGE, v_page=2 * PAGE),
    _joint(2 * HEAD, k_token=128, v_token=128, k_head=128 * 16, v_head=128 * 16, k_page=2 * PAGE, v_page=2 * PAGE),
    # a column range of wider rows, V's a page later too
    _joint(2 * 128 + 2 * 16 * 512, k_token=512, v_token=512, k_head=64, v_head=64, k_page=16 * 512, v_page=16 * 512),
])
def test_keys_and_values_may_share_a_buffer(lib, change):
    for fn in ("swam_cache_append", "swam_cache_attention"):
        assert _call(lib, fn, change) == (INVALID, "ctx is NULL"), fn


def test_the_overlap_of_keys_and_values_is_found_exactly(lib):
    """Random shifts of layouts with the same strides, against the elements themselves."""
    rng = random.Random(3)
    seen = [0, 0]
    for _ in range(400):
        n = [rng.randint(1, 3), 8, rng.randint(1, 3)]             # pages, tokens, heads
        order, step, steps = rng.sample(range(3), 3), 64, [0] * 3
        for i in order:                                           # the closest first, some with room between
            step += 8 * rng.choice([0, 0, 8, 24])
            steps[i] = step
            step *= n[i]
        heads = {p * steps[0] + t * steps[1] + h * steps[2] for p in range(n[0]) for t in range(8) for h in range(n[2])}
        shift = 8 * rng.randint(-step // 8 - 8, step // 8 + 8)
        if shift == 0:
            continue
        # two head vectors meet where their starts are less than one apart
        meet = any(s + shift + x in heads for s in heads for x in range(-56, 64, 8))
        rc, msg = _call(lib, "swam_cache_append", {
            "cache.k": _p(10), "cache.v": _p(10) + 2 * shift, "cache.n_pages": n[0], "cache.page_size": 8, "cache.n_kv_heads": n[2],
            "cache.k_page": steps[0], "cache.k_token": steps[1], "cache.k_head": steps[2], "cache.v_page": steps[0],
            "cache.v_token": steps[1], "cache.v_head": steps[2], "ks": 256, "vs": 256})
        assert (rc, msg) == (INVALID, "the cache's k and v overlap" if meet else "ctx is NULL"), (n, steps, shift)
        seen[meet] += 1
    assert min(seen) > 50
