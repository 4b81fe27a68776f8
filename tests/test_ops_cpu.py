"""Host-side checks of the operators of swam_ops.h (no GPU): exports, and every
refusal.  A call is checked before its context, so a NULL context shows what is
wrong with the call itself; fake pointers are never dereferenced."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE, UNSUPPORTED = -1, -2, -7


@pytest.fixture(scope="module")
def lib():
    from paper_2609_38984_amd import swam
    if not os.path.exists(swam.LIB_PATH):
        from paper_2609_38984_amd.build import build
        build()
    return swam.load_library()


def test_every_declared_operator_is_exported(lib):
    from paper_2609_38984_amd import swam
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "swam_ops.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(swam_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(swam.OP_EXPORTS)
    for n in names:
        assert hasattr(lib, n), n
    for name, value in re.findall(r"#define SWAM_(I8_MAX_WIDTH|I8_MAX_K|GEMM_GELU)\s+(\d+)", text):
        assert getattr(swam, name) == int(value)


def _p(i):
    """A pointer of its own 64 GB range, 256-byte aligned."""
    return (i + 1) << 36


NORM = dict(x=_p(0), xs=64, res=_p(1), rs=64, gain=_p(2), shift=_p(3), scale=_p(4), eps=1e-6, rows=8, d=64,
            sum=_p(5), ss=64, q=_p(6), qs=64, qsc=_p(7))
QUANT = dict(x=_p(0), xs=64, rows=8, d=64, q=_p(6), qs=64, qsc=_p(7))
GEMM = dict(a=_p(0), lda=64, asc=_p(1), b=_p(2), ldb=64, bsc=_p(3), bias=_p(4), res=_p(5), ldr=32, gate=_p(6),
            flags=0, c=_p(7), ldc=32, m=8, n=32, k=64)
ATTN = dict(q=_p(0), qs=256, k=_p(1), ks=128, v=_p(2), vs=128, mask=_p(3), cu_q=_p(4), cu_k=_p(5), kv=_p(6),
            n_seqs=2, n_kv=3, n_q=10, n_k=20, heads=4, kv_heads=2, dim=64, scale=0.125, o=_p(7), os=256,
            lse=_p(8))


def _call(lib, fn, base, change):
    a = dict(base)
    a.update(change)
    rc = getattr(lib, fn)(None, *a.values())
    return rc, lib.swam_last_error(None).decode()


@pytest.mark.parametrize("fn,base", [("swam_rms_norm_i8", NORM), ("swam_quantize_i8", QUANT),
                                     ("swam_gemm_i8", GEMM), ("swam_cross_attention", ATTN)])
def test_a_good_call_only_lacks_its_context(lib, fn, base):
    assert _call(lib, fn, base, {}) == (INVALID, "ctx is NULL")


@pytest.mark.parametrize("change,code,word", [
    (dict(rows=-1), INVALID, "rows"), (dict(rows=1 << 31), SHAPE, "rows"),
    (dict(d=0), SHAPE, "WIDTH"), (dict(d=32769, xs=40000, qs=40000), SHAPE, "WIDTH"),
    (dict(x=None), INVALID, "required"), (dict(q=None), INVALID, "required"), (dict(qsc=None), INVALID, "required"),
    (dict(xs=63), INVALID, "stride"), (dict(qs=63), INVALID, "stride"), (dict(qs=-64), INVALID, "stride"),
    (dict(x=_p(0) + 1), INVALID, "aligned"), (dict(qsc=_p(7) + 2), INVALID, "aligned"),
    (dict(q=_p(0)), INVALID, "overlaps"), (dict(q=_p(0) + 1023), INVALID, "overlaps"),
    (dict(qsc=_p(6) + 64), INVALID, "overlaps"), (dict(qsc=_p(0) + 512), INVALID, "overlaps"),
])
def test_row_quantiser_refuses(lib, change, code, word):
    for fn, base in (("swam_quantize_i8", QUANT), ("swam_rms_norm_i8", NORM)):
        rc, msg = _call(lib, fn, base, change)
        assert rc == code and word in msg, (fn, msg)


@pytest.mark.parametrize("change,code,word", [
    (dict(rs=63), INVALID, "stride"), (dict(ss=10), INVALID, "stride"),
    (dict(shift=None), INVALID, "together"), (dict(scale=None), INVALID, "together"),
    (dict(eps=-1e-6), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"),
    (dict(res=_p(1) + 1), INVALID, "aligned"), (dict(gain=_p(2) + 1), INVALID, "aligned"),
    (dict(shift=_p(3) + 2), INVALID, "aligned"), (dict(sum=_p(5) + 1), INVALID, "aligned"),
    (dict(sum=_p(0) + 2), INVALID, "sum_out"),          # a row of x later by one element
    (dict(sum=_p(0), ss=128), INVALID, "sum_out"),      # the same start at another stride
    (dict(sum=_p(1) + 128), INVALID, "sum_out"),
    (dict(sum=_p(2) - 64), INVALID, "sum_out"),         # runs into gain
    (dict(q=_p(5) + 8), INVALID, "overlaps"), (dict(q=_p(3)), INVALID, "overlaps"),
])
def test_rms_norm_refuses(lib, change, code, word):
    rc, msg = _call(lib, "swam_rms_norm_i8", NORM, change)
    assert rc == code and word in msg, msg


def test_rms_norm_takes_the_sum_in_place_and_beside(lib):
    for change in (dict(sum=_p(0)), dict(sum=_p(1)), dict(res=None, sum=_p(0)), dict(sum=None),
                   dict(xs=128, ss=128, sum=_p(0) + 128)):      # the other half of x's rows
        assert _call(lib, "swam_rms_norm_i8", NORM, change) == (INVALID, "ctx is NULL"), change


@pytest.mark.parametrize("change,code,word", [
    (dict(m=-1), INVALID, "m and n"), (dict(n=-1), INVALID, "m and n"), (dict(m=1 << 30), SHAPE, "2^30"),
    (dict(k=0), SHAPE, "multiple of 16"), (dict(k=56), SHAPE, "multiple of 16"),
    (dict(k=131072, lda=131072, ldb=131072), SHAPE, "multiple of 16"),
    (dict(flags=2), INVALID, "flags"), (dict(flags=1), UNSUPPORTED, "GELU"),
    (dict(res=None), INVALID, "gate"),
    (dict(a=None), INVALID, "required"), (dict(asc=None), INVALID, "required"), (dict(b=None), INVALID, "required"),
    (dict(bsc=None), INVALID, "required"), (dict(c=None), INVALID, "required"),
    (dict(lda=48), INVALID, "stride"), (dict(ldb=48), INVALID, "stride"), (dict(ldc=31), INVALID, "stride"),
    (dict(ldr=31), INVALID, "stride"), (dict(lda=1 << 22), SHAPE, "2^22"), (dict(ldb=1 << 23), SHAPE, "2^22"),
    (dict(a=_p(0) + 8), INVALID, "16-byte"), (dict(b=_p(2) + 4), INVALID, "16-byte"),
    (dict(lda=72), INVALID, "16-byte"), (dict(ldb=65), INVALID, "16-byte"),
    (dict(asc=_p(1) + 2), INVALID, "element type"), (dict(bias=_p(4) + 1), INVALID, "element type"),
    (dict(c=_p(7) + 1), INVALID, "element type"),
    (dict(c=_p(0)), INVALID, "overlaps an input"), (dict(c=_p(4) + 32), INVALID, "overlaps an input"),
    (dict(c=_p(6)), INVALID, "overlaps an input"), (dict(c=_p(5) + 2), INVALID, "residual"),
    (dict(c=_p(5), ldc=64), INVALID, "residual"),
])
def test_gemm_refuses(lib, change, code, word):
    rc, msg = _call(lib, "swam_gemm_i8", GEMM, change)
    assert rc == code and word in msg, msg


def test_gemm_takes_its_residual_in_place_and_a_column_range(lib):
    for change in (dict(c=_p(5)), dict(ldr=64, ldc=64, c=_p(5) + 64), dict(k=131056, lda=131056, ldb=131056),
                   dict(res=None, gate=None, flags=1), dict(bias=None, gate=None),
                   dict(m=0, a=None, c=None), dict(n=0, ldc=0, ldr=0, b=None)):
        assert _call(lib, "swam_gemm_i8", GEMM, change) == (INVALID, "ctx is NULL"), change


@pytest.mark.parametrize("change,code,word", [
    (dict(dim=32), SHAPE, "head_dim"), (dict(dim=96), SHAPE, "head_dim"),
    (dict(heads=0), INVALID, "n_heads"), (dict(heads=5), INVALID, "n_heads"), (dict(kv_heads=0), INVALID, "n_heads"),
    (dict(n_seqs=0), SHAPE, "sequences"), (dict(n_seqs=65), SHAPE, "sequences"), (dict(n_kv=65), SHAPE, "sequences"),
    (dict(n_kv=0), SHAPE, "sequences"),
    (dict(cu_q=None), INVALID, "cu_q"), (dict(cu_k=None), INVALID, "cu_k"), (dict(kv=None), INVALID, "kv_seq"),
    (dict(scale=0.0), INVALID, "scale"), (dict(scale=-1.0), INVALID, "scale"),
    (dict(scale=float("inf")), INVALID, "scale"), (dict(scale=float("nan")), INVALID, "scale"),
    (dict(n_q=-1), INVALID, "n_q"), (dict(n_k=-1), INVALID, "n_q"),
    (dict(n_q=1 << 28), SHAPE, "2^30"), (dict(n_k=1 << 30), SHAPE, "2^30"),
    (dict(q=None), INVALID, "required"), (dict(o=None), INVALID, "required"), (dict(k=None), INVALID, "required"),
    (dict(v=None), INVALID, "required"),
    (dict(qs=255), INVALID, "stride"), (dict(os=128), INVALID, "stride"), (dict(ks=120), INVALID, "stride"),
    (dict(vs=0), INVALID, "stride"), (dict(ks=1 << 22), SHAPE, "2^22"),
    (dict(q=_p(0) + 8), INVALID, "16-byte"), (dict(k=_p(1) + 2), INVALID, "16-byte"), (dict(ks=132), INVALID, "16-byte"),
    (dict(os=260), INVALID, "16-byte"),
    (dict(lse=_p(8) + 1), INVALID, "element type"), (dict(cu_q=_p(4) + 2), INVALID, "element type"),
    (dict(o=_p(0) + 512), INVALID, "overlaps an input"), (dict(o=_p(1)), INVALID, "overlaps an input"),
    (dict(lse=_p(3)), INVALID, "overlaps an input"), (dict(lse=_p(7) + 512), INVALID, "o overlaps lse"),
])
def test_cross_attention_refuses(lib, change, code, word):
    rc, msg = _call(lib, "swam_cross_attention", ATTN, change)
    assert rc == code and word in msg, msg


def test_cross_attention_takes_empty_and_interleaved_tensors(lib):
    for change in (dict(n_q=0, q=None, o=None), dict(n_k=0, k=None, v=None, ks=0, vs=0),
                   dict(ks=256, vs=256, v=_p(1) + 256),             # K and V side by side
                   dict(qs=512, os=512, o=_p(0) + 512),             # o beside q in one buffer
                   dict(n_seqs=64, n_kv=64, kv=None), dict(n_seqs=1, n_kv=1, cu_q=None, cu_k=None, kv=None),
                   dict(mask=None, lse=None)):
        assert _call(lib, "swam_cross_attention", ATTN, change) == (INVALID, "ctx is NULL"), change


@pytest.mark.parametrize("fn,base,name,rows", [
    ("swam_quantize_i8", QUANT, "xs", 8), ("swam_quantize_i8", QUANT, "qs", 8), ("swam_rms_norm_i8", NORM, "rs", 8),
    ("swam_rms_norm_i8", NORM, "ss", 8), ("swam_gemm_i8", GEMM, "ldc", 8), ("swam_gemm_i8", GEMM, "ldr", 8)])
def test_rows_that_no_memory_holds_are_refused(lib, fn, base, name, rows):
    for far in ((1 << 48) // rows + 1, 1 << 62):
        rc, msg = _call(lib, fn, base, {name: far})
        assert rc == SHAPE and "2^48" in msg, msg
    # one row has no second to reach
    one = {"rows": 1} if "rows" in base else {"m": 1}
    assert _call(lib, fn, base, {name: 1 << 62, **one}) == (INVALID, "ctx is NULL")
