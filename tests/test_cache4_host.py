"""Host-side checks of include/hqmq_cache4.h that need no GPU: what the library exports, sizes, refusals before anything is
enqueued (pointers here are addresses that are never read), and the plain form's own properties."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import cache4_cpp
import cache4_ref as ref
from cache4_plan import plan
import paper_2605_27646_amd as hq
from paper_2605_27646_amd import cache4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 40  # aligned addresses
INVALID, UNSUPPORTED, SMALL = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hq.library_path()):
        from paper_2605_27646_amd import build
        build.build()
    return cache4._load()


def test_header_and_library_agree(lib):
    header = open(os.path.join(ROOT, "include", "hqmq_cache4.h")).read()
    declared = set(re.findall(r"^(?:int32_t|uint64_t)\s+(hqmq_\w+)\s*\(", header, re.M))
    assert declared == {"hqmq_cache4_sizes", "hqmq_cache4_write", "hqmq_cache4_read", "hqmq_cache4_attend",
                        "hqmq_cache4_attend_workspace_bytes"}
    for name in declared:
        assert hasattr(lib, name) and hasattr(hq, name), name
    for name in ("HQMQ_CACHE4_FLOAT", "HQMQ_CACHE4_INT"):
        assert int(re.search(rf"#define {name} (\d+)", header).group(1)) == getattr(hq, name)
    assert (C.sizeof(cache4.Cache4Params), C.sizeof(cache4._Buffers), C.sizeof(cache4._Batch), C.sizeof(cache4._Rows)) == (20, 32, 40, 24)


def _params(**kw):
    d = dict(n_pages=100, page_size=16, H=4, D=128, format=0)
    d.update(kw)
    return hq.Cache4Params(*d.values())


@pytest.mark.parametrize("D,groups", [(1, 1), (32, 1), (33, 2), (96, 3), (100, 4), (128, 4), (129, 6), (192, 6), (193, 8), (256, 8)])
@pytest.mark.parametrize("fmt", [0, 1])
def test_sizes(lib, D, groups, fmt):
    assert hq.hqmq_cache4_sizes(_params(D=D, format=fmt)) == (100 * 16 * 4 * groups * 16, 100 * 16 * 4 * groups * (4 if fmt else 1))
    pages = ref.Pages(100, 16, 4, D, fmt)
    assert (pages.k.size, pages.ks.size, pages.v.size, pages.vs.size) == hq.hqmq_cache4_sizes(_params(D=D, format=fmt)) * 2


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(n_pages=0)), (INVALID, dict(n_pages=-1)), (INVALID, dict(page_size=8)), (INVALID, dict(page_size=48)), (INVALID, dict(page_size=1 << 21)),
    (INVALID, dict(H=0)), (UNSUPPORTED, dict(H=4097)), (INVALID, dict(D=0)), (UNSUPPORTED, dict(D=257)), (UNSUPPORTED, dict(format=2)),
    (UNSUPPORTED, dict(format=-1)), (UNSUPPORTED, dict(n_pages=2 ** 31 - 1, page_size=1 << 20, H=4096)),
])
def test_sizes_refuse(lib, want, kw):
    a, b = C.c_uint64(), C.c_uint64()
    assert lib.hqmq_cache4_sizes(C.byref(_params(**kw)), C.byref(a), C.byref(b)) == want
    assert _call(lib, "write", **{"params": _params(**kw)}) == want
    with pytest.raises(hq.HqmqError):
        hq.alloc_cache4(_params(**kw), "cpu")


def _rows(data=P + (5 << 30), row=512, head=128):
    return cache4._Rows(data, row, head)


def _call(lib, what, params=None, cache=None, n_seqs=3, pages=10, max_rows=8, max_length=160, table=P, lengths=P, starts=P, n_rows=24, heads=8, type=0,
          a=None, b=None, scale=0.1, window=0, lse=0, ws=P, ws_bytes=1 << 40):
    params = params or _params()
    cache = cache if cache is not None else cache4._Buffers(P, P + (1 << 30), P + (2 << 30), P + (3 << 30))
    batch = cache4._Batch(n_seqs, pages, max_rows, max_length, table, lengths, starts or None)
    if what == "attend":
        a, b = a or _rows(row=1024), b or _rows(P + (6 << 30), row=1024)
        return lib.hqmq_cache4_attend(C.byref(params), C.byref(cache), C.byref(batch), n_rows, heads, type, C.byref(a), scale, window, C.byref(b), lse or None, ws,
                                      ws_bytes, None)
    a, b = a or _rows(), b or _rows(P + (6 << 30))
    return getattr(lib, "hqmq_cache4_" + what)(C.byref(params), C.byref(cache), C.byref(batch), n_rows, type, C.byref(a), C.byref(b), None)


@pytest.mark.parametrize("what", ["write", "read", "attend"])
@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(n_seqs=0)), (INVALID, dict(n_seqs=-1)), (UNSUPPORTED, dict(n_seqs=65536)), (INVALID, dict(pages=0)), (UNSUPPORTED, dict(pages=1 << 27)),
    (INVALID, dict(max_rows=0)), (INVALID, dict(max_length=0)), (INVALID, dict(n_rows=-1)), (INVALID, dict(starts=0, n_rows=25)),
    (INVALID, dict(table=None)), (INVALID, dict(lengths=None)), (INVALID, dict(table=P + 2)), (INVALID, dict(lengths=P + 1)), (INVALID, dict(starts=P + 3)),
    (UNSUPPORTED, dict(type=2)), (UNSUPPORTED, dict(type=-1)), (UNSUPPORTED, dict(n_rows=(1 << 30) + 1)),
    (INVALID, dict(cache=cache4._Buffers(None, P, P, P))), (INVALID, dict(cache=cache4._Buffers(P, P + 4096, P + (2 << 30), P + (3 << 30)))),
    (INVALID, dict(cache=cache4._Buffers(P, P + (1 << 30), P, P + (3 << 30)))), (INVALID, dict(cache=cache4._Buffers(P + 8, P + (1 << 30), P + (2 << 30), P + (3 << 30)))),
    (INVALID, dict(cache=cache4._Buffers(P, P + (1 << 30), P + (2 << 30), P + (1 << 30) + 16))),
    (INVALID, dict(a=_rows(None))), (INVALID, dict(b=_rows(None))), (INVALID, dict(a=_rows(P + 1))), (INVALID, dict(a=_rows(row=-1))), (INVALID, dict(b=_rows(head=-128))),
    (UNSUPPORTED, dict(a=_rows(row=1 << 31))),
])
def test_calls_refuse(lib, what, want, kw):
    assert _call(lib, what, **kw) == want


@pytest.mark.parametrize("what", ["read", "attend"])
@pytest.mark.parametrize("row,head", [(512, 127), (512, 0), (0, 128), (384, 128), (100, 1 << 20), (128, 128 * 23)])
def test_rows_that_share_elements_are_not_written(lib, what, row, head):
    assert _call(lib, what, b=_rows(row=row, head=head)) == INVALID


def test_read_refuses_one_place_for_both(lib):
    assert _call(lib, "read", a=_rows(), b=_rows()) == INVALID


@pytest.mark.parametrize("b", [
    _rows(P + (5 << 30) + 2),                 # the second channel on
    _rows(P + (5 << 30) + 2 * 512 * 23),      # the last row is the first
    _rows(P + (5 << 30) - 2 * 512 * 5),       # shifted by some rows
    _rows(P + (5 << 30) + 2 * 127),           # the last channel of a head
    _rows(P + (5 << 30) + 2 * (512 + 64), row=1024),  # other strides in the same memory
])
def test_read_refuses_rows_that_share_elements(lib, b):
    assert _call(lib, "read", a=_rows(), b=b) == INVALID
    assert _call(lib, "read", a=b, b=_rows()) == INVALID


@pytest.mark.parametrize("what", ["write", "read", "attend"])
@pytest.mark.parametrize("which", ["a", "b"])
@pytest.mark.parametrize("buffer", range(4))
@pytest.mark.parametrize("at", ["first", "last", "around"])
def test_rows_over_the_cache_are_refused(lib, what, which, buffer, at):
    """Rows that begin inside one of the cache's buffers, end inside it, or enclose it."""
    sizes = hq.hqmq_cache4_sizes(_params())
    base, n = P + (buffer << 30), sizes[buffer % 2]
    row = 1024 if what == "attend" else 512
    heads = 8 if what == "attend" else 4
    extent = 2 * (23 * row + (heads - 1) * 128 + 128)
    rows = {"first": _rows(base + n - 2, row=row), "last": _rows(base - extent + 2, row=row), "around": _rows(base - 4096, row=(n + 8192) // 2)}[at]
    assert _call(lib, what, **{which: rows}) == INVALID


@pytest.mark.parametrize("b", [
    _rows(P + (5 << 30) + 2 * 1024, row=1024),          # the result of a row over the next row's queries
    _rows(P + (5 << 30) - 2 * 1024 * 20, row=1024),
    _rows(P + (5 << 30) + 2 * 128, row=1024),           # over the next head's
    _rows(P + (5 << 30) + 2, row=1024),
    _rows(P + (5 << 30), row=1024 + 128),               # from the same place on, with other strides
])
def test_attend_refuses_results_over_other_queries(lib, b):
    assert _call(lib, "attend", a=_rows(row=1024), b=b) == INVALID


SHARE = """
extern "C" int share(uint64_t a, uint64_t b, int64_t a_row, int64_t a_head, int64_t b_row, int64_t b_head, int n, int heads, int D)
{
    const hqmq_cache4_rows x = {reinterpret_cast<void *>(a), a_row, a_head}, y = {reinterpret_cast<void *>(b), b_row, b_head};
    return cache4_rows_share(&x, &y, n, heads, D);
}
"""


def test_rows_that_share_elements_are_found(tmp_path):
    """Against sets of elements: rows beside each other in one tensor share none, shifted ones do; never missed with other strides."""
    code = cache4_cpp.between("hqmq_api.hip", "static uint64_t cache4_extent", "static bool cache4_rows_over_cache")
    code += cache4_cpp.between("hqmq_api.hip", "static bool cache4_same_strides", "\nstatic Cache4Seqs") + SHARE
    host = cache4_cpp.compiled(tmp_path, code)
    host.share.argtypes = [C.c_uint64] * 2 + [C.c_int64] * 4 + [C.c_int] * 3
    rng = np.random.default_rng(0)
    elements = lambda at, row, head, n, heads, D: {at + i * row + j * head + c for i in range(n) for j in range(heads) for c in range(D)}
    seen = set()
    for _ in range(4000):
        n, heads, D = (int(x) for x in rng.integers(1, 5, 3))
        strides = []
        for _ in range(2):
            inner = D + int(rng.integers(0, 2 * D + 2))
            if rng.random() < 0.5:  # heads in rows, or rows in heads
                head, row = inner, (heads - 1) * inner + D + int(rng.integers(0, 3 * D))
            else:
                row, head = inner, (n - 1) * inner + D + int(rng.integers(0, 3 * D))
            strides.append((row, head))
        if rng.random() < 0.8:
            strides[1] = strides[0]
        a, b = 1000, 1000 + int(rng.integers(-60, 60))
        one, other = elements(a, *strides[0], n, heads, D), elements(b, *strides[1], n, heads, D)
        got = bool(host.share(2 * a, 2 * b, *strides[0], *strides[1], n, heads, D))
        shared, apart = bool(one & other), min(one) > max(other) or min(other) > max(one)
        same = all(count == 1 or x == y for count, x, y in zip((n, heads), *strides))
        if shared or apart or same:
            assert got == shared, (n, heads, D, strides, b - a)
        else:
            assert got  # other strides in the same memory are not looked at one by one
        seen.add((shared, apart, same))
    assert len(seen) == 6  # what is apart shares nothing
    far = 1 << 45  # the largest strides and counts
    assert not host.share(far, far + 2 * 128, 1 << 30, 1 << 8, 1 << 30, 1 << 8, 1 << 30, 2, 128)
    assert host.share(far, far + 2 * ((1 << 59) + 127), 1 << 30, 1 << 8, 1 << 30, 1 << 8, 1 << 30, 2, 128)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(heads=0)), (INVALID, dict(heads=6)), (INVALID, dict(heads=-4)), (UNSUPPORTED, dict(heads=65536)), (INVALID, dict(window=-1)),
    (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (UNSUPPORTED, dict(scale=-2.0 ** 101)), (INVALID, dict(lse=P + 2)), (INVALID, dict(ws=P + 128)),
    (INVALID, dict(ws=None)), (SMALL, dict(ws_bytes=100)), (UNSUPPORTED, dict(n_rows=1 << 29)),
])
def test_attend_refuses(lib, want, kw):
    kw = dict(dict(max_length=160000, pages=10000), **kw)
    assert _call(lib, "attend", **kw) == want


def test_calls_without_rows_enqueue_nothing(lib):
    for what in ("write", "read", "attend"):
        assert _call(lib, what, n_rows=0, a=_rows(None), b=_rows(None), ws=None, ws_bytes=0) == 0
        assert _call(lib, what, n_rows=0, table=None) == INVALID


def test_attend_workspace(lib):
    table, lengths = torch.zeros(1, 4096, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    params = _params(n_pages=4096, H=8)
    long = hq.Cache4Batch(table, lengths, max_length=65536)
    n = hq.hqmq_cache4_attend_workspace_bytes(params, long, 1, 32)
    assert n > 0 and _call(lib, "attend", params=params, n_seqs=1, pages=4096, max_length=65536, starts=0, n_rows=1, heads=32, ws_bytes=n - 1) == SMALL
    assert hq.hqmq_cache4_attend_workspace_bytes(params, hq.Cache4Batch(table, lengths, max_length=100), 1, 32) == 0
    assert hq.hqmq_cache4_attend_workspace_bytes(params, long, 1, 32, window=64) == 0
    assert hq.hqmq_cache4_attend_workspace_bytes(params, long, 1, 31) == 0 and hq.hqmq_cache4_attend_workspace_bytes(_params(D=300), long, 1, 32) == 0
    # what the table has room for is what counts where the hint is larger
    assert hq.hqmq_cache4_attend_workspace_bytes(params, hq.Cache4Batch(table, lengths), 1, 32) == n


@pytest.mark.parametrize("n_seqs,n_rows", [(1, 4096), (1, 100000), (3, 12000), (64, 4160), (5000, 9000), (2, 3)])
@pytest.mark.parametrize("H,G,D", [(8, 4, 128), (1, 1, 256), (2, 16, 64), (32, 1, 200)])
def test_attend_workspace_with_too_few_rows_believed(lib, n_seqs, n_rows, H, G, D):
    """A batch of more rows than max_rows allows for is cut by the rows that there are.  Tokens are split for fewer workgroups than 256
    compute units, into at most 512 / workgroups parts (or 256 / workgroups, if that is more), and a workgroup has at most 64 rows, so
    there are 512 * 64 partial rows at most, of all channels in fp32, a reference and a sum."""
    table, lengths, starts = (torch.zeros(shape, dtype=torch.int32) for shape in ((n_seqs, 2048), (n_seqs,), (n_seqs + 1,)))
    params = _params(n_pages=4096, H=H, D=D)
    width = ref.width_of(D)
    bytes_of = lambda **hints: hq.hqmq_cache4_attend_workspace_bytes(params, hq.Cache4Batch(table, lengths, starts, **hints), n_rows, H * G)
    for max_length in (300, 5000, 32768):
        for max_rows in (1, 7, 100):
            n = bytes_of(max_rows=max_rows, max_length=max_length)
            assert n <= 512 * 64 * (4 * width + 8) + 256
            if n_seqs == 1:  # all rows are its own, whatever is believed
                assert n == bytes_of(max_rows=n_rows, max_length=max_length)


def test_attend_plan_of_too_few_rows_believed(lib):
    """One sequence of 4096 rows is cut the same way whatever max_rows says; of several, by the rows that they have on average."""
    right = plan(8, 128, 64, 1, 512, 4096, 32, max_rows=4096, max_length=32768)
    assert (right.blocks, right.n_tiles, right.n_splits) == (4, 256, 1)
    for believed in (1, 100, 4095):
        assert plan(8, 128, 64, 1, 512, 4096, 32, max_rows=believed, max_length=32768) == right
    assert plan(8, 128, 64, 4, 512, 4096, 32, max_rows=1) == plan(8, 128, 64, 4, 512, 4096, 32, max_rows=1024) == plan(8, 128, 64, 4, 512, 4096, 32, starts=False)
    # what is believed rightly is left as it is: a step of 64 sequences, and one with a prompt
    assert plan(8, 128, 16, 64, 512, 64, 32, max_rows=1)[:3] == (1, 1, 1) and plan(8, 128, 16, 64, 512, 63 + 2048, 32, max_rows=2048).blocks == 4


def test_binding_refuses_shapes(lib):
    i32 = dict(dtype=torch.int32)
    table, lengths = torch.zeros(2, 5, **i32), torch.zeros(2, **i32)
    for bad in ((table[0], lengths), (table.long(), lengths), (table, lengths[:1]), (table.t(), lengths), (table, lengths, torch.zeros(2, **i32)),
                (table, lengths, torch.zeros(3))):
        with pytest.raises(ValueError):
            hq.Cache4Batch(*bad)
    batch, params = hq.Cache4Batch(table, lengths), _params()
    cache = hq.alloc_cache4(params, "cpu")
    k = torch.zeros(4, 4, 128, dtype=torch.float16)
    for kk, vv in ((k.float(), k.float()), (k[:, :3], k), (k, k[:2]), (k, k.bfloat16()), (k[0], k), (torch.zeros(4, 4, 129, dtype=torch.float16)[:, :, :-1].transpose(1, 2), k),
                   (torch.zeros(4, 4, 256, dtype=torch.float16)[:, :, ::2], k)):
        for call in (hq.hqmq_cache4_write, hq.hqmq_cache4_read):
            with pytest.raises(ValueError):
                call(params, cache, batch, kk, vv)
    q = torch.zeros(4, 8, 128, dtype=torch.float16)
    for kw in (dict(out=q[:, :4]), dict(out=q.bfloat16()), dict(q=q.float()), dict(lse=torch.zeros(4, 7)), dict(workspace=torch.zeros(4, 4).t())):
        args = dict(q=q, out=q, workspace=None, lse=None)
        args.update(kw)
        with pytest.raises(ValueError):
            hq.hqmq_cache4_attend(params, cache, batch, args["q"], 1.0, args["out"], args["workspace"], lse=args["lse"])
    for field in ("k_codes", "k_scales", "v_codes", "v_scales"):
        short = hq.alloc_cache4(params, "cpu")
        setattr(short, field, getattr(short, field)[:-1])
        with pytest.raises(ValueError, match="hold"):
            hq.hqmq_cache4_write(params, short, batch, k, k.clone())


@pytest.mark.parametrize("field", ["k_codes", "k_scales", "v_codes", "v_scales"])
@pytest.mark.parametrize("dtype", [torch.int8, torch.float16, torch.int32])
def test_buffers_are_bytes(lib, field, dtype):
    """A tensor of another type, a key of 16-bit numbers say, is not taken for pages, however many bytes it has."""
    params = _params()
    k = torch.zeros(4, 4, 128, dtype=torch.float16)
    batch = hq.Cache4Batch(torch.zeros(2, 5, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    cache = hq.alloc_cache4(params, "cpu")
    setattr(cache, field, torch.zeros(1 << 20, dtype=dtype))
    for call in (lambda: hq.hqmq_cache4_write(params, cache, batch, k, k.clone()), lambda: hq.hqmq_cache4_read(params, cache, batch, k, k.clone()),
                 lambda: hq.hqmq_cache4_attend(params, cache, batch, k, 1.0, k.clone())):
        with pytest.raises(ValueError, match="uint8"):
            call()


def test_binding_counts_of_more_than_32_bits(lib):
    table, lengths = torch.zeros(1, 4096, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    params = _params(n_pages=4096, H=8)
    bytes_of = lambda window=0, **hints: hq.hqmq_cache4_attend_workspace_bytes(params, hq.Cache4Batch(table, lengths, **hints), 1, 32, window=window)
    assert bytes_of(window=2 ** 32 + 1) == bytes_of(window=2 ** 30) and bytes_of(max_rows=2 ** 32 + 1, max_length=2 ** 32 + 1) == bytes_of() > 0
    assert bytes_of(window=-2 ** 32) == 0
    cache, batch = hq.alloc_cache4(_params(), "cpu"), hq.Cache4Batch(table, lengths)
    for many in (torch.zeros(1, 4, 128, dtype=torch.float16).expand(2 ** 32 + 1, 4, 128), torch.zeros(1, 1, 128, dtype=torch.float16).expand(1, 2 ** 32 + 4, 128)):
        with pytest.raises(ValueError, match="2.31"):
            hq.hqmq_cache4_write(_params(), cache, batch, many, many)
        with pytest.raises(ValueError, match="2.31"):
            hq.hqmq_cache4_attend(_params(), cache, batch, many, 1.0, many)


def test_binding_sizes_of_more_than_32_bits(lib):
    """A number of rows, heads, pages or anything else that 32 bits do not hold is no number that they would hold."""
    table, lengths = torch.zeros(1, 4096, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    params, batch = _params(n_pages=4096, H=8), hq.Cache4Batch(table, lengths)
    assert hq.hqmq_cache4_attend_workspace_bytes(params, batch, 1, 32) > 0
    for rows, heads in ((2 ** 32 + 1, 32), (1, 2 ** 32 + 32), (1 - 2 ** 32, 32), (2 ** 31, 32)):
        assert hq.hqmq_cache4_attend_workspace_bytes(params, batch, rows, heads) == 0
    for name in ("n_pages", "page_size", "H", "D", "format"):
        for value in (2 ** 32 + 16, -2 ** 32 + 16, 2 ** 31):
            with pytest.raises(ValueError, match="32 bits"):
                _params(**{name: value})
            with pytest.raises(ValueError, match="32 bits"):
                setattr(params, name, value)
    assert hq.hqmq_cache4_sizes(params) == hq.hqmq_cache4_sizes(_params(n_pages=4096, H=8))
    with pytest.raises(ValueError, match="32 bits"):
        hq.Cache4Params(n_pages=2 ** 32 + 100, page_size=16, H=8, D=128, format=0)


DIVIDED = """
// The first number that is divided wrongly, the largest factor, and the largest product with it; beside every multiple of d, and at the ends.
extern "C" int64_t check(uint32_t from, uint32_t to, uint64_t *mul, uint64_t *product)
{
    constexpr uint64_t kEnd = 1ull << 30;
    for (uint32_t d = from; d <= to; ++d) {
        const Divisor by = make_divisor(d);
        *mul = std::max<uint64_t>(*mul, by.mul);
        *product = std::max(*product, (kEnd - 1) * by.mul);
        const uint64_t multiples = (kEnd - 1) / d, stride = multiples / 3000 + 1;
        for (uint64_t k = 0; k <= multiples; k += k < 64 || k + 64 > multiples ? 1 : stride)
            for (uint64_t n = k * d == 0 ? 0 : k * d - 1; n <= k * d + 1 && n < kEnd; ++n)
                if ((uint64_t)divided((int)n, by) != n / d)
                    return (int64_t)n;
        if ((uint64_t)divided((int)(kEnd - 1), by) != (kEnd - 1) / d)
            return (int64_t)kEnd - 1;
    }
    return -1;
}
"""


def test_division_by_multiplication(tmp_path):
    """Every divisor that there is (query heads of a kv head, dwords of a row, parts of the tokens), numbers up to 2^30 - 1 where a quotient
    changes; and the sizes that the proof names: a factor of at most 2^31, products below 2^61."""
    host = cache4_cpp.compiled(tmp_path, cache4_cpp.between("hqmq_cache4_device.h", "struct Divisor {", "// What no kernel writes") + DIVIDED)
    host.check.restype, host.check.argtypes = C.c_int64, [C.c_uint32, C.c_uint32, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]
    mul, product = C.c_uint64(), C.c_uint64()
    for first, last in ((1, 300), (32767, 32770), (65000, 65535)):
        assert host.check(first, last, C.byref(mul), C.byref(product)) == -1
    assert 2 ** 30 + 1 < mul.value <= 2 ** 31 and product.value < 2 ** 61


PLACES = """
#include <cstdio>
#include <initializer_list>
#define __device__
#define __forceinline__ inline
%s
int main()
{
    for (int NG : {1, 2, 3, 4, 6, 8})
        for (int w = 0; w < 4 * NG; ++w)
            for (int t = 0; t < 4; ++t) {
                const Cache4Place p = cache4_v_place(NG, w, t);
                for (int r = 0; r < p.runs; ++r)
                    for (int b = 0; b < p.bytes; ++b)
                        printf("%%d %%d %%d %%d %%d\\n", NG, t, 8 * w + 2 * (r * p.bytes + b), p.at + r * 4 * p.bytes + b, p.runs * p.bytes);
            }
}
"""


def test_places_of_v(tmp_path):
    """The kernels' address of every byte of V, compiled for the host, against the plain form's."""
    source = open(os.path.join(ROOT, "paper_2605_27646_amd", "csrc", "hqmq_cache4_device.h")).read()
    start, end = source.index("struct Cache4Place {"), source.index("// ---- launches")
    code = tmp_path / "places.cpp"
    code.write_text(PLACES % ("#include <cstdint>\n" + source[start:end]))
    subprocess.run(["g++", "-std=c++17", "-o", str(tmp_path / "places"), str(code)], check=True)
    out = subprocess.run([str(tmp_path / "places")], check=True, capture_output=True, text=True).stdout
    rows = np.array([[int(x) for x in line.split()] for line in out.splitlines()])
    assert (rows[:, 4] == 4).all()
    for NG in (1, 2, 3, 4, 6, 8):
        pages = ref.Pages(1, 16, 1, 32 * NG, 0)
        mine = rows[rows[:, 0] == NG]
        assert len(mine) == 4 * 16 * NG and len(set(mine[:, 3])) == len(mine)  # a place of its own for each
        for t in range(4):
            of = mine[mine[:, 1] == t]
            assert np.array_equal(of[np.argsort(of[:, 2])][:, 3], pages._v_bytes(t))


@pytest.mark.parametrize("fmt", [0, 1])
def test_plain_form_is_within_half_a_step(fmt):
    """What comes back is the nearest value that the group's scale allows."""
    x = np.random.default_rng(fmt).standard_normal((50, 96)).astype(np.float16).astype(np.float64)
    codes, scales = ref.quantise(fmt, x)
    y = ref.dequantise(fmt, codes, scales, 96)
    if fmt == 0:
        unit = np.repeat(2.0 ** (scales[..., 0].astype(float) - 127), 32, -1)
        gap = np.where(np.abs(x) <= 2 * unit, 0.25, np.where(np.abs(x) <= 4 * unit, 0.5, 1.0)) * unit  # 4 to 7 may be off by one unit
        assert (np.abs(x - y) <= gap).all() and (scales[..., 0] >= 104).all() and (scales[..., 0] <= 140).all()
    else:
        step = np.repeat(np.ascontiguousarray(scales).view(np.float16)[..., 0].astype(float), 32, -1)
        # half a step, 15 times the rounding of the step to fp16, and that of the value
        assert (np.abs(x - y) <= step * (0.5 + 15 * 2.0 ** -11) + 2.0 ** -11 * np.abs(y)).all()
