"""The paged 4-bit cache on the GPU: rows written, read back and attended to, against the plain numpy form (cache4_ref.py)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import cache4_ref as ref
import paper_2605_27646_amd as hq

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
HALF = {F16: 2.0 ** -11, BF16: 2.0 ** -8}      # half a step, relative
WEIGHT = {F16: 2.0 ** -22, BF16: 2.0 ** -11}   # of the softmax weights in the products with V
FMT = [hq.HQMQ_CACHE4_FLOAT, hq.HQMQ_CACHE4_INT]


def _np(t):
    return t.detach().cpu().double().numpy()


class World:
    """A cache with its plain copy, its sequences' pages in random order; unwritten bytes hold 0xFF (NaN scales)."""

    def __init__(self, seed, fmt, H, D, page, n_seqs, pages_per_seq, spare=2, fill=0xFF):
        rng = np.random.default_rng(seed)
        self.rng, self.H, self.D, self.page, self.fmt = rng, H, D, page, fmt
        n_pages = n_seqs * pages_per_seq + spare
        self.params = hq.Cache4Params(n_pages, page, H, D, fmt)
        self.plain = ref.Pages(n_pages, page, H, D, fmt, fill)
        self.cache = hq.alloc_cache4(self.params, DEV)
        self.buffers = (self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales)
        for t in self.buffers:
            t.fill_(fill)
        self.table = rng.permutation(n_pages)[:n_seqs * pages_per_seq].reshape(n_seqs, pages_per_seq).astype(np.int32)
        self.n_seqs = n_seqs

    def batch(self, lengths, rows=None, **hints):
        """rows: numbers of rows per sequence (None: equal shares)."""
        starts = None
        if rows is not None:
            starts = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device=DEV)
        return hq.Cache4Batch(torch.tensor(self.table, device=DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), starts, **hints)

    def places(self, lengths, rows):
        """(row, sequence, position) of every row of the call."""
        row = 0
        for i, n in enumerate(rows):
            length = min(max(lengths[i], 0), self.table.shape[1] * self.page)
            for j in range(n):
                yield row, i, length - n + j
                row += 1

    def write_plain(self, lengths, rows, k, v):
        for role, x in enumerate((k, v)):
            codes, scales = ref.quantise(self.fmt, _np(x))
            for row, i, pos in self.places(lengths, rows):
                if pos >= 0:
                    p = int(self.table[i, pos // self.page])
                    if 0 <= p < self.plain.n_pages:
                        self.plain.put(role, p, pos % self.page, codes[row], scales[row])

    def same_bytes(self):
        torch.cuda.synchronize()
        for got, want in zip(self.buffers, (self.plain.k, self.plain.ks, self.plain.v, self.plain.vs)):
            got = got.cpu().numpy().reshape(want.shape)
            bad = np.argwhere(got != want)
            assert bad.size == 0, (bad[:4], got[tuple(bad[0])], want[tuple(bad[0])], len(bad))

    def fill_random(self, lengths, dtype, gain=1.0, hot=False):
        """Every sequence's tokens written by the library and by the plain form."""
        n = int(sum(lengths))
        k, v = (self.values(n, dtype, gain, hot and role == 0) for role in range(2))
        hq.hqmq_cache4_write(self.params, self.cache, self.batch(lengths, lengths), k, v)
        self.write_plain(lengths, lengths, k, v)

    def values(self, n, dtype, gain=1.0, hot=False, heads=None):
        x = self.rng.standard_normal((n, heads or self.H, self.D)) * gain
        if hot:
            x[:, :, 3::32] *= 8
        return torch.tensor(x, dtype=dtype, device=DEV)


def _check_attend(w, lengths, rows, dtype, G, scale=None, window=0, starts=True, gain=1.5, poison=True, strided=False, **hints):
    Hq, n = w.H * G, int(sum(rows))
    scale = w.D ** -0.5 if scale is None else scale
    batch = w.batch(lengths, rows if starts else None, **hints)
    q = w.values(n, dtype, gain, heads=Hq)
    if strided:  # the middle of a wider projection, heads before rows in the result
        wide = torch.full((n, Hq + 3, w.D + 5), 9.0, dtype=dtype, device=DEV)
        wide[:, 1:Hq + 1, 2:w.D + 2] = q
        q = wide[:, 1:Hq + 1, 2:w.D + 2]
        out = torch.full((Hq, n, w.D + 1), float("nan"), dtype=dtype, device=DEV)[:, :, :w.D].transpose(0, 1)
    else:
        out = torch.full((n, Hq, w.D), float("nan"), dtype=dtype, device=DEV)
    lse = torch.full((n, Hq), float("nan"), device=DEV)
    ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, n, Hq, window) + 256, dtype=torch.uint8, device=DEV)
    if poison:
        ws.fill_(0xFF)
    hq.hqmq_cache4_attend(w.params, w.cache, batch, q, scale, out, ws, window=window, lse=lse)
    torch.cuda.synchronize()
    got, got_lse, qn = _np(out), _np(lse), _np(q)
    at = list(w.places(lengths, rows))
    worst = 0.0
    for i in range(w.n_seqs):
        mine = [(row, pos) for row, seq, pos in at if seq == i]
        if not mine:
            continue
        idx, pos = np.array([m[0] for m in mine]), np.array([m[1] for m in mine])
        length = min(max(lengths[i], 0), w.table.shape[1] * w.page)
        k, there = w.plain.sequence(0, w.table[i], length)
        v, _ = w.plain.sequence(1, w.table[i], length)
        o, l, tol, tol_l = ref.attend(qn[idx], k, v, there, pos, scale, window, HALF[dtype], WEIGHT[dtype])
        err = np.abs(got[idx] - o)
        assert np.isfinite(got[idx]).all(), (i, lengths[i])
        assert (err <= tol).all(), (i, lengths[i], rows[i], np.argwhere(err > tol)[:3], (err / tol).max())
        worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
        seen = np.isfinite(l)
        assert (got_lse[idx][~seen] == -np.inf).all() and (got[idx][~seen] == 0).all()
        err = np.abs(got_lse[idx][seen] - l[seen])
        assert (err <= tol_l[seen]).all(), (i, (err / tol_l[seen]).max())
    return out, lse, worst


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,H,page", [(128, 3, 16), (64, 2, 64), (96, 5, 16), (256, 1, 32), (1, 1, 16), (33, 2, 16), (100, 3, 32), (130, 2, 16), (200, 1, 128)])
def test_rows_written_and_read_back(fmt, dtype, D, H, page):
    """Byte for byte; slots without a row keep what they held; rows of no sequence are left as they were."""
    w = World(D + page, fmt, H, D, page, 4, 3 if page < 64 else 2)
    lengths, rows = [2 * page, 7, page + 5, 1], [2 * page, 0, page - 2, 1]
    k, v = (w.values(sum(rows) + 3, dtype, hot=role == 0) for role in range(2))
    batch = w.batch(lengths, rows)
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()
    back = [torch.full_like(x, float("nan")) for x in (k, v)]
    hq.hqmq_cache4_read(w.params, w.cache, batch, *back)
    torch.cuda.synchronize()
    for role, x in enumerate(back):
        assert torch.isnan(x[sum(rows):]).all()
        for row, i, pos in w.places(lengths, rows):
            want = torch.tensor(w.plain.get(role, int(w.table[i, pos // page]), pos % page)).to(dtype)
            assert torch.equal(x[row].cpu(), want), (role, row)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_write_of_unusual_values(fmt, dtype):
    """Zeros of both signs, the smallest numbers, ties, infinities, NaN, numbers beyond the largest, groups of one value."""
    w = World(5, fmt, 2, 64, 16, 1, 4)
    n = 40
    x = w.rng.standard_normal((n, 2, 64))
    x[0] = 0.0
    x[1] = -0.0
    x[2] = 3.25
    x[3, :, :32] = np.array([6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5] * 2)
    x[3, :, 32:] = np.arange(32) / 2 - 3
    x[4] *= 2.0 ** -24
    x[5] *= 2.0 ** -20
    x[6] *= 30000
    x[7, 0, 5], x[7, 1, 40] = np.inf, -np.inf
    x[8, 0, 7], x[8, 1, 33] = np.nan, np.nan
    x[9] = np.where(np.arange(64) % 2, 65504.0, -65504.0)
    x[10] = 1000 + x[10] / 8
    x[11, :, 1:32] = 0
    x[12] = 7.0
    x[13] = np.nextafter(np.float16(7.0), np.float16(8.0))
    x[14] = np.nan
    x[15] = np.arange(64) % 16 * 1.5 + 0.75 * (np.arange(64) % 3 == 0)
    for i in range(16, n):
        x[i] = np.round(x[i] * 4) / 4 * 2.0 ** (i - 28)
    k = torch.tensor(x, dtype=dtype, device=DEV)
    v = torch.tensor(x[::-1].copy(), dtype=dtype, device=DEV)
    hq.hqmq_cache4_write(w.params, w.cache, w.batch([n], [n]), k, v)
    w.write_plain([n], [n], k, v)
    w.same_bytes()
    back = [torch.empty_like(k) for _ in range(2)]
    hq.hqmq_cache4_read(w.params, w.cache, w.batch([n]), *back)
    assert all(torch.isfinite(b).all() for b in back)


@pytest.mark.parametrize("fmt", FMT)
def test_many_groups_near_ties(fmt):
    """A large odd batch with strides of its own, every code and scale the same as the plain form's."""
    w = World(9, fmt, 3, 100, 32, 3, 40)
    lengths, rows = [1280, 901, 77], [1280, 515, 77]
    wide = torch.tensor(w.rng.standard_normal((sum(rows), 7, 108)) * 3, dtype=F16, device=DEV)
    k, v = wide[:, 1:4, 3:103], wide[:, 4:, 8:]
    hq.hqmq_cache4_write(w.params, w.cache, w.batch(lengths, rows, max_rows=16), k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()


def test_tokens_without_a_place():
    """Pages that are none, lengths beyond the table and below zero, more rows than tokens."""
    w = World(11, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 5, 3)
    w.table[0, 1], w.table[1, 0], w.table[2, 2] = -1, w.params.n_pages, 2 ** 31 - 1
    lengths, rows = [48, 20, 1000, 3, -7], [40, 20, 48, 9, 2]
    k, v = (w.values(sum(rows), F16) for _ in range(2))
    batch = w.batch(lengths, rows)
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()
    back = [torch.full_like(k, float("nan")) for _ in range(2)]
    hq.hqmq_cache4_read(w.params, w.cache, batch, *back)
    torch.cuda.synchronize()
    for row, i, pos in w.places(lengths, rows):
        p = int(w.table[i, pos // 16]) if pos >= 0 else -1
        for role in range(2):
            want = w.plain.get(role, p, pos % 16) if 0 <= p < w.params.n_pages else np.zeros((2, 64))
            assert np.array_equal(_np(back[role][row]), want), (row, i, pos)
    # whole tokens of the sequences, some of them missing, unwritten ones with finite bytes
    w = World(12, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 5, 3)
    w.fill_random([48] * 5, F16)
    w.table[0, 1], w.table[1, 0], w.table[2, 2] = -1, w.params.n_pages, 2 ** 31 - 1
    for rows in ([40, 20, 48, 9, 2], [1] * 5):
        _check_attend(w, lengths, rows, F16, 2)
        _check_attend(w, lengths, rows, F16, 2, window=18)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [128, 64, 96, 32, 192, 256, 100, 17, 130])
@pytest.mark.parametrize("rows", [1, 5, 40])
def test_attend_every_kernel(fmt, dtype, D, rows):
    """Every form of the kernel: format, type, width, and 16, 32 or 64 query rows of a workgroup."""
    w = World(3 * D + rows, fmt, 2, D, 16, 3, 10)
    lengths = [150, rows, 97]
    w.fill_random(lengths, dtype, hot=True)
    _check_attend(w, lengths, [rows] * 3, dtype, 3)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 513])
@pytest.mark.parametrize("page", [16, 64])
def test_attend_lengths(length, page):
    w = World(length, hq.HQMQ_CACHE4_FLOAT, 2, 128, page, 2, -(-length // page))
    lengths = [length, max(1, length - 1)]
    w.fill_random(lengths, F16)
    _check_attend(w, lengths, [1, 1], F16, 4, starts=False)
    _check_attend(w, lengths, lengths, F16, 2)


@pytest.mark.parametrize("window", [1, 2, 16, 31, 33, 100, 300, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("rows,G", [(1, 4), (7, 4), (90, 1)])
def test_attend_windows(window, rows, G):
    w = World(window % 1000 + rows, hq.HQMQ_CACHE4_INT, 2, 64, 16, 2, 32)
    lengths = [500, 333]
    w.fill_random(lengths, BF16)
    _check_attend(w, lengths, [rows, min(rows, 50)], BF16, G, window=window)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("rows,window", [(1, 33), (1, 100), (6, 50), (40, 17)])
def test_what_no_row_sees_may_hold_anything(fmt, rows, window):
    """Pages before the windows given back: none, or one that holds another's bytes, here NaN scales; the same behind the last row."""
    w = World(rows + window, fmt, 2, 96, 16, 2, 24)
    lengths = [300, 187]
    w.fill_random(lengths, F16)
    other = [p for p in range(w.params.n_pages) if p not in set(w.table.ravel())][0]  # never written
    plain = w.table.copy()
    for i, length in enumerate(lengths):
        given_back = max(0, length - rows + 1 - window) // 16
        w.table[i, :given_back:2], w.table[i, 1:given_back:2] = other, -1
        w.table[i, -(-length // 16):] = other
    out, lse, _ = _check_attend(w, lengths, [rows, rows], F16, 3, window=window)
    w.table = plain
    w.rng = np.random.default_rng(0)
    want = _check_attend(w, lengths, [rows, rows], F16, 3, window=window)
    w.table[:, :1] = other
    w.rng = np.random.default_rng(0)
    got = _check_attend(w, lengths, [rows, rows], F16, 3, window=window)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_starts_that_do_not_ascend():
    """Rows are lost, or some are computed twice, but every access stays inside the tensors: both ways of dealing places."""
    w = World(77, hq.HQMQ_CACHE4_FLOAT, 4, 64, 16, 80, 4)
    w.fill_random([64] * 80, F16)
    n = 700
    k, v, q = w.values(n, F16), w.values(n, F16), w.values(n, F16, heads=16)
    out, ws = torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        starts = torch.randint(-50, n + 50, (81,), generator=g).to(torch.int32).to(DEV)
        lengths = torch.randint(-5, 80, (80,), generator=g).to(torch.int32).to(DEV)
        for hint in (1, n):
            batch = hq.Cache4Batch(torch.tensor(w.table, device=DEV), lengths, starts, max_rows=hint)
            hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
            hq.hqmq_cache4_read(w.params, w.cache, batch, k.clone(), v.clone())
            hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws)
    torch.cuda.synchronize()


class Fenced:
    """Tensors in the middle of larger ones; whole() says whether what lies around them is as it was."""

    def __init__(self):
        self.all = []

    def tensor(self, *shape, dtype):
        item = torch.empty(0, dtype=dtype).element_size()
        n, margin = int(np.prod(shape)) * item, 1 << 16
        whole = torch.full((n + 2 * margin,), 0xA5, dtype=torch.uint8, device=DEV)
        self.all.append((whole, margin, n))
        return whole[margin:margin + n].view(dtype).view(shape)

    def whole(self):
        return all(bool((t[:m] == 0xA5).all()) and bool((t[m + n:] == 0xA5).all()) for t, m, n in self.all)


@pytest.mark.parametrize("fmt,dtype,D", [(hq.HQMQ_CACHE4_FLOAT, F16, 64), (hq.HQMQ_CACHE4_INT, BF16, 100)])
@pytest.mark.parametrize("pages", [4, 80])
def test_starts_that_do_not_ascend_reach_nothing_else(fmt, dtype, D, pages):
    """Every tensor that the calls write lies between others: what is around them, and pages of no sequence, keep their bytes, with places of each
    sequence and along all rows, with tokens in parts and whole."""
    n_seqs, H, n, spare = 80 if pages == 4 else 6, 4, 700 if pages == 4 else 12, 3
    rng = np.random.default_rng(pages)
    params = hq.Cache4Params(n_seqs * pages + spare, 16, H, D, fmt)
    fence = Fenced()
    cache = hq.Cache4Buffers(*(fence.tensor(size, dtype=torch.uint8) for size in hq.hqmq_cache4_sizes(params) * 2))
    buffers = (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)
    order = rng.permutation(params.n_pages)
    table, unused = torch.tensor(order[:-spare].reshape(n_seqs, pages).astype(np.int32), device=DEV), torch.tensor(order[-spare:], device=DEV)
    for t in buffers:
        t.zero_()
        t.view(params.n_pages, -1)[unused] = 0x5A
    out, back_k, back_v = (fence.tensor(n, heads, D, dtype=dtype) for heads in (16, H, H))
    lse = fence.tensor(n, 16, dtype=torch.float32)
    make = lambda heads: torch.tensor(rng.standard_normal((n, heads, D)), dtype=dtype, device=DEV)
    k, v, q = make(H), make(H), make(16)
    seen = set()
    for seed in range(6):
        g = torch.Generator().manual_seed(seed)
        starts = torch.randint(-50, n + 50, (n_seqs + 1,), generator=g).to(torch.int32).to(DEV)
        lengths = torch.randint(-5, 16 * pages + 16, (n_seqs,), generator=g).to(torch.int32).to(DEV)
        for hint in (1, n):
            batch = hq.Cache4Batch(table, lengths, starts, max_rows=hint)
            ws = fence.tensor(max(256, hq.hqmq_cache4_attend_workspace_bytes(params, batch, n, 16)), dtype=torch.uint8)
            seen.add(ws.numel() > 256)
            hq.hqmq_cache4_write(params, cache, batch, k, v)
            hq.hqmq_cache4_read(params, cache, batch, back_k, back_v)
            hq.hqmq_cache4_attend(params, cache, batch, q, 0.1, out, ws, lse=lse)
            assert fence.whole(), (seed, hint)
            assert all(bool((t.view(params.n_pages, -1)[unused] == 0x5A).all()) for t in buffers), (seed, hint)
    assert seen == {pages == 80}


@pytest.mark.parametrize("hint", [1, 200, 1024, 2048, 2 ** 30])
@pytest.mark.parametrize("rows", [1, 20])
def test_attend_splits_and_hints(hint, rows):
    """Few and many splits of the tokens, whatever the host believes of lengths and rows."""
    w = World(hint % 997, hq.HQMQ_CACHE4_FLOAT, 1, 128, 32, 2, 64)
    lengths = [2048, 700]
    w.fill_random(lengths, F16)
    a = _check_attend(w, lengths, [rows, rows // 2], F16, 4, max_length=hint, max_rows=rows)
    _check_attend(w, lengths, [rows, rows // 2], F16, 4, max_length=hint, max_rows=1)
    assert a[0].dtype == F16


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("scale", [0.0, -0.2, 2.0, 1e-30, 30.0])
def test_attend_scales(fmt, scale):
    """Uniform weights, negative scales, and scores of which one takes all the weight, later ones larger."""
    w = World(21, fmt, 2, 64, 16, 2, 20)
    lengths = [300, 129]
    w.fill_random(lengths, F16, hot=True)
    _check_attend(w, lengths, [3, 70], F16, 2, scale=scale)


@pytest.mark.parametrize("dtype,gain", [(BF16, 1e-20), (BF16, 1e20), (F16, 2.0 ** -20), (F16, 5000.0)])
def test_attend_queries_of_any_size(dtype, gain):
    w = World(31, hq.HQMQ_CACHE4_FLOAT, 1, 128, 16, 2, 8)
    lengths = [100, 64]
    w.fill_random(lengths, dtype)
    _check_attend(w, lengths, [2, 2], dtype, 4, gain=gain, scale=0.1 / gain)


@pytest.mark.parametrize("D,G,rows", [(96, 5, 13), (100, 1, 3), (128, 16, 2), (33, 33, 2)])
def test_attend_strides_and_groups(D, G, rows):
    w = World(D + G, hq.HQMQ_CACHE4_INT, 3, D, 32, 3, 5)
    lengths = [160, 33, rows]
    w.fill_random(lengths, F16)
    _check_attend(w, lengths, [rows, 1, rows], F16, G, strided=True)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 6, 7, 9, 11, 31, 36, 63, 95, 125, 135, 190, 250, 255])
def test_heads_that_end_anywhere(fmt, dtype, D):
    """Every number of last channels, in every width: rows between others that are not read nor written, at odd addresses."""
    w = World(D, fmt, 2, D, 16, 2, 3)
    lengths, rows = [37, 18], [21, 18]
    n = sum(rows)
    wide = w.values(n + 2, dtype, heads=2 * (2 * D + 3))[:, :, 0].contiguous() * 1000  # [n + 2, 2 (2 D + 3)], channels beside the rows' own
    k, v = ((wide[1:-1, 1 + i * D:] if i else wide[1:-1, 1:])[:, :2 * (D + 1)].unflatten(1, (2, D + 1))[:, :, :D] for i in range(2))
    batch = w.batch(lengths, rows)
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()
    back = [torch.full((n, 2, D + 3), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
    hq.hqmq_cache4_read(w.params, w.cache, batch, *(x[:, :, 1:D + 1] for x in back))
    tight = [torch.empty(n, 2, D, dtype=dtype, device=DEV) for _ in range(2)]
    hq.hqmq_cache4_read(w.params, w.cache, batch, *tight)
    for role, (x, y) in enumerate(zip(back, tight)):
        assert torch.equal(x[:, :, 1:D + 1], y) and (x[:, :, 0] == 7).all() and (x[:, :, D + 1:] == 7).all()
        for i, (length, first) in enumerate(zip(lengths, (0, 21))):
            z, there = w.plain.sequence(role, w.table[i], length)
            z = torch.tensor(z[length - rows[i]:], dtype=torch.float64).to(dtype)
            assert torch.equal(y[first:first + rows[i]].cpu(), z)
    w = World(D + 1, fmt, 2, D, 16, 2, 3)
    w.fill_random(lengths, dtype)
    _check_attend(w, lengths, rows, dtype, 3, strided=True)


def test_attend_rising_scores():
    """Keys whose scores grow along the sequence, so that the reference is renewed again and again."""
    w = World(41, hq.HQMQ_CACHE4_FLOAT, 1, 32, 16, 1, 64)
    n = 1000
    k = torch.zeros(n, 1, 32, dtype=F16, device=DEV)
    k[:, 0, 0] = torch.linspace(-300, 300, n).half()
    v = w.values(n, F16)
    hq.hqmq_cache4_write(w.params, w.cache, w.batch([n], [n]), k, v)
    w.write_plain([n], [n], k, v)
    for gain in (0.2, -1.0):
        q = torch.full((1, 2, 32), gain, dtype=F16, device=DEV)
        out, lse = torch.empty_like(q), torch.empty(1, 2, device=DEV)
        ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
        hq.hqmq_cache4_attend(w.params, w.cache, w.batch([n]), q, 1.0, out, ws, lse=lse)
        kk, there = w.plain.sequence(0, w.table[0], n)
        vv, _ = w.plain.sequence(1, w.table[0], n)
        o, l, tol, tol_l = ref.attend(_np(q), kk, vv, there, np.array([n - 1]), 1.0, 0, HALF[F16], WEIGHT[F16])
        assert (np.abs(_np(out) - o) <= tol).all() and (np.abs(_np(lse) - l) <= tol_l).all()


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype,size", [(F16, 2.0 ** -6), (F16, 60000.0), (BF16, 2.0 ** -6), (BF16, 2.0 ** 90), (BF16, 2.0 ** 127)])
@pytest.mark.parametrize("scale", [2.0 ** 24, -1.0, 2.0 ** 60, 2.0 ** 100])
def test_scores_of_any_size(fmt, dtype, size, scale):
    """A token whose score is far above the others' has all the weight, two that tie have halves, whatever the scores are."""
    w = World(43, fmt, 1, 64, 16, 2, 40)
    n = 600
    k = torch.zeros(2 * n, 1, 64, dtype=dtype, device=DEV)
    k[:, 0, 0] = -4 if scale < 0 else 4
    k[torch.arange(0, 2 * n, 3), 0, 0] = -1
    for token in (99, n + 7, n + 599):
        k[token, 0, 0] = -6 if scale < 0 else 6
    v = w.values(2 * n, dtype)
    hq.hqmq_cache4_write(w.params, w.cache, w.batch([n, n], [n, n]), k, v)
    w.write_plain([n, n], [n, n], k, v)
    q = torch.zeros(4, 3, 64, dtype=dtype, device=DEV)
    q[:, :, 0] = size
    q[0, 1, 0], q[3, 1, 0] = 0.5, 0.25
    for hint in (600, 1):  # split or not
        batch = w.batch([n, n], [1, 3], max_length=hint)
        out, lse = torch.empty_like(q), torch.empty(4, 3, device=DEV)
        ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, scale, out, ws, lse=lse)
        got, got_lse = _np(out), _np(lse)
        for row, (seq, tokens) in enumerate([(0, [99]), (1, [7]), (1, [7]), (1, [7, 599])]):
            vv, _ = w.plain.sequence(1, w.table[seq], n)
            kk, _ = w.plain.sequence(0, w.table[seq], n)
            want = vv[tokens, 0].mean(0)
            for head in range(3):
                x = float(q[row, head, 0])
                s = float(np.float32(scale)) * x * kk[tokens[0], 0, 0]
                gap = s - float(np.float32(scale)) * x * kk[300 if seq else 100, 0, 0]
                assert np.isfinite(got[row, head]).all()
                if abs(gap) < 200 or max(abs(s), abs(float(np.float32(scale)) * x)) > 2.0 ** 126:  # others have weight as well
                    continue
                # 2^-20: sums of two weights, their reciprocal and what rounding the values leaves
                assert (np.abs(got[row, head] - want) <= np.abs(want) * (HALF[dtype] + 2.0 ** -20) + 2.0 ** -25).all(), (row, head)
                assert abs(got_lse[row, head] - s) <= abs(s) * 2.0 ** -21 + 1, (row, head)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,hint", [(1, 600), (1, 1), (9, 600), (40, 1)])
def test_queries_that_are_not_finite(fmt, dtype, rows, hint):
    """They give NaN where they see a token, zeros where they see none, and nothing to other rows."""
    w = World(44, fmt, 2, 64, 16, 3, 40)
    lengths = [600, 300, 0]
    w.fill_random(lengths, dtype)
    q = w.values(3 * rows, dtype, heads=6)
    batch = w.batch(lengths, [rows] * 3, max_length=hint)
    ws = torch.full((1 << 24,), 0xFF, dtype=torch.uint8, device=DEV)
    results = []
    lost = torch.zeros(3 * rows, 6, dtype=torch.bool)
    for turn in range(2):
        out, lse = torch.empty_like(q), torch.empty(3 * rows, 6, device=DEV)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.125, out, ws, lse=lse)
        results.append((out.cpu(), lse.cpu()))
        if turn == 0:
            for row in range(0, 3 * rows, 2 if rows > 1 else 1):
                value = [float("nan"), float("inf"), -float("inf")][row % 3]
                q[row, row % 6, (7 * row) % 64] = value
                lost[row, row % 6] = True
    (a, la), (b, lb) = results
    empty = torch.arange(3 * rows)[:, None].expand(-1, 6) >= 2 * rows
    assert torch.equal(a[~lost], b[~lost]) and torch.equal(la[~lost], lb[~lost])
    assert b[lost & ~empty].isnan().all() and lb[lost & ~empty].isnan().all()
    assert (b[empty] == 0).all() and (lb[empty] == -float("inf")).all()


def test_steps_together():
    """As a server runs them: prompts written in chunks and attended to, then token by token with drafts taken back; every step's
    attention and the cache's bytes the same as the plain form's."""
    w = World(51, hq.HQMQ_CACHE4_FLOAT, 2, 128, 16, 3, 8)
    lengths = np.array([0, 0, 0])
    for rows in ([40, 0, 17], [30, 64, 1], [1, 1, 1], [5, 3, 0], [1, 1, 1], [2, 1, 4]):
        lengths = lengths + rows
        k, v = (w.values(sum(rows), BF16, hot=role == 0) for role in range(2))
        batch = w.batch(lengths.tolist(), rows, max_rows=max(rows))
        hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
        w.write_plain(lengths.tolist(), rows, k, v)
        _check_attend(w, lengths.tolist(), rows, BF16, 4, max_rows=max(rows))
        if rows == [5, 3, 0]:
            lengths = lengths - [3, 3, 0]  # rejected drafts: their slots are written again
    w.same_bytes()


@pytest.mark.parametrize("fmt,dtype", [(hq.HQMQ_CACHE4_FLOAT, BF16), (hq.HQMQ_CACHE4_INT, F16)])
def test_one_prompt_among_many_steps(fmt, dtype):
    """A batch of which one sequence has nearly all rows: places along all rows instead of the largest sequence's for each."""
    n = 70
    w = World(55, fmt, 4, 64, 32, n, 20)
    rows = [1] * n
    rows[0], rows[13], rows[40], rows[69] = 0, 600, 37, 0
    lengths = [int(x) for x in w.rng.integers(1, 90, n)]
    lengths[13], lengths[40] = 640, 37
    k, v = (w.values(sum(rows), dtype) for _ in range(2))
    w.fill_random(lengths, dtype)
    batch = w.batch(lengths, rows, max_rows=600)
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()
    back = [torch.full_like(x, float("nan")) for x in (k, v)]
    hq.hqmq_cache4_read(w.params, w.cache, batch, *back)
    for row, i, pos in w.places(lengths, rows):
        want = torch.tensor(w.plain.get(0, int(w.table[i, pos // 32]), pos % 32)).to(dtype)
        assert torch.equal(back[0][row].cpu(), want), row
    _check_attend(w, lengths, rows, dtype, 4, max_rows=600, max_length=640)
    _check_attend(w, lengths, rows, dtype, 4, max_rows=1, max_length=640)


@pytest.mark.parametrize("fmt,dtype", [(hq.HQMQ_CACHE4_FLOAT, BF16), (hq.HQMQ_CACHE4_INT, F16)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ragged", [False, True])
def test_one_head_of_many_rows(fmt, dtype, D, ragged):
    """A shard of a model: one kv head, thousands of rows, in one sequence or most of them in one of many."""
    n = 40 if ragged else 1
    w = World(D + n, fmt, 1, D, 64, n, 66)
    rows = [3] * n
    rows[n // 2] = 4101
    lengths = [int(x) for x in w.rng.integers(3, 100, n)]
    lengths[n // 2] = 4201
    k, v = (w.values(sum(rows), dtype, hot=role == 0) for role in range(2))
    batch = w.batch(lengths, rows)
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()
    back = [torch.full_like(x, float("nan")) for x in (k, v)]
    hq.hqmq_cache4_read(w.params, w.cache, batch, *back)
    back = [_np(x) for x in back]
    for row, i, pos in w.places(lengths, rows):
        for role in range(2):
            want = torch.tensor(w.plain.get(role, int(w.table[i, pos // 64]), pos % 64)).to(dtype).double().numpy()
            assert np.array_equal(back[role][row], want), (row, role)


def test_thousands_of_sequences():
    """Most of them with one row, some with none, one with many: three rounds of the search for a place's sequence."""
    n = 5000
    w = World(57, hq.HQMQ_CACHE4_FLOAT, 1, 32, 16, n, 2)
    rows = [int(x) for x in w.rng.integers(0, 2, n)]
    rows[17], rows[4999] = 32, 5
    lengths = [max(r, int(x)) for r, x in zip(rows, w.rng.integers(0, 33, n))]
    k, v = (w.values(sum(rows), F16) for _ in range(2))
    batch = w.batch(lengths, rows)  # what a sequence may have is not known: all rows
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    w.write_plain(lengths, rows, k, v)
    w.same_bytes()
    for t in w.buffers[1::2]:  # unwritten scales are zeros from here on
        t[t == 255] = 0
    w.plain.ks[w.plain.ks == 255] = 0
    w.plain.vs[w.plain.vs == 255] = 0
    _check_attend(w, lengths, rows, F16, 2)


def test_no_rows():
    w = World(61, hq.HQMQ_CACHE4_INT, 2, 64, 16, 2, 2)
    none = torch.empty(0, 2, 64, dtype=F16, device=DEV)
    for batch in (w.batch([5, 0]), w.batch([5, 0], [0, 0])):
        hq.hqmq_cache4_write(w.params, w.cache, batch, none, none)
        hq.hqmq_cache4_read(w.params, w.cache, batch, none, none.clone())
        hq.hqmq_cache4_attend(w.params, w.cache, batch, none, 1.0, none)
        assert hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, 0, 2) == 0
    w.same_bytes()


def test_tensors_elsewhere_are_refused():
    """Each tensor of the three calls in turn in host memory."""
    w = World(79, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 2, 40)
    here = w.batch([600, 500])
    host = hq.Cache4Batch(*(t.cpu() for t in here._tensors[:2]))
    k, q = w.values(2, F16), w.values(2, F16)
    args = dict(cache=w.cache, batch=here, k=k, v=k.clone(), q=q, out=torch.empty_like(q), ws=torch.empty(1 << 22, dtype=torch.uint8, device=DEV),
                lse=torch.empty(2, 2, device=DEV))
    elsewhere = {name: x.cpu() for name, x in args.items() if isinstance(x, torch.Tensor)}
    elsewhere.update(batch=host, cache=hq.alloc_cache4(w.params, "cpu"))
    for name, x in elsewhere.items():
        a = dict(args, **{name: x})
        if name not in ("q", "out", "ws", "lse"):
            for call in (hq.hqmq_cache4_write, hq.hqmq_cache4_read):
                with pytest.raises(ValueError, match="current device"):
                    call(w.params, a["cache"], a["batch"], a["k"], a["v"])
        if name not in ("k", "v"):
            with pytest.raises(ValueError, match="current device"):
                hq.hqmq_cache4_attend(w.params, a["cache"], a["batch"], a["q"], 0.1, a["out"], a["ws"], lse=a["lse"])
    mixed = hq.alloc_cache4(w.params, DEV)
    mixed.v_scales = mixed.v_scales.cpu()
    with pytest.raises(ValueError, match="one device"):
        hq.hqmq_cache4_write(w.params, mixed, here, k, k.clone())
    with pytest.raises(ValueError, match="one device"):
        hq.Cache4Batch(here._tensors[0], here._tensors[1].cpu())


def test_buffers_set_anew():
    """Calls follow a Cache4Buffers whose tensors are replaced, and other params of the same buffers."""
    w, other = World(80, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 1, 4), World(81, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 1, 4)
    k, v = w.values(20, F16), w.values(20, F16)
    hq.hqmq_cache4_write(w.params, w.cache, w.batch([20], [20]), k, v)
    w.write_plain([20], [20], k, v)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        setattr(w.cache, name, getattr(other.cache, name))
    k, v = w.values(30, F16), w.values(30, F16)
    hq.hqmq_cache4_write(other.params, w.cache, other.batch([30], [30]), k, v)
    other.write_plain([30], [30], k, v)
    w.same_bytes()
    other.same_bytes()
    small = hq.Cache4Params(other.params.n_pages, 16, 1, 64, hq.HQMQ_CACHE4_FLOAT)  # half the heads
    one = World(82, hq.HQMQ_CACHE4_FLOAT, 1, 64, 16, 1, 4)
    other.cache.k_codes.fill_(0xFF), other.cache.k_scales.fill_(0xFF), other.cache.v_codes.fill_(0xFF), other.cache.v_scales.fill_(0xFF)
    k, v = one.values(9, BF16), one.values(9, BF16)
    hq.hqmq_cache4_write(small, w.cache, one.batch([9], [9]), k, v)
    one.write_plain([9], [9], k, v)
    one.buffers = tuple(t[:t.numel() // 2] for t in other.buffers)
    one.same_bytes()


def test_expanded_rows_are_read():
    """One row for all tokens, one head for all heads: strides of 0."""
    w = World(83, hq.HQMQ_CACHE4_INT, 4, 96, 16, 2, 4)
    k = w.values(1, F16, heads=1).expand(50, 4, 96)
    v = w.values(50, F16, heads=1).expand(50, 4, 96)
    hq.hqmq_cache4_write(w.params, w.cache, w.batch([27, 23], [27, 23]), k, v)
    w.write_plain([27, 23], [27, 23], k, v)
    w.same_bytes()
    with pytest.raises(hq.HqmqError):  # but not written
        hq.hqmq_cache4_read(w.params, w.cache, w.batch([27, 23], [27, 23]), k, v)
    with pytest.raises(hq.HqmqError):
        hq.hqmq_cache4_attend(w.params, w.cache, w.batch([27, 23], [27, 23]), v, 0.1, v, torch.empty(1 << 20, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("fmt", FMT)
def test_rows_beside_each_other(fmt):
    """K and V read into one memory between each other: by rows, by heads, by channels, by role; into places that overlap they are not."""
    w = World(84, fmt, 3, 40, 16, 2, 4)
    lengths = [60, 21]
    w.fill_random(lengths, F16)
    n = sum(lengths)
    want = [np.concatenate([w.plain.sequence(role, w.table[i], length)[0] for i, length in enumerate(lengths)]) for role in range(2)]
    fused = lambda *shape: torch.full(shape, 7.0, dtype=F16, device=DEV)
    a, b, c, d = fused(n, 2, 3, 40), fused(n, 3, 2, 40), fused(n, 3, 83), fused(2, 3, n, 40)
    views = [(a[:, 0], a[:, 1]), (b[:, :, 1], b[:, :, 0]), (c[:, :, :40], c[:, :, 43:]), (d[0].transpose(0, 1), d[1].transpose(0, 1)),
             (a.view(n, 6, 40)[:, ::2], a.view(n, 6, 40)[:, 1::2])]
    for k, v in views:
        hq.hqmq_cache4_read(w.params, w.cache, w.batch(lengths, lengths), k, v)
        assert np.array_equal(_np(k), want[0]) and np.array_equal(_np(v), want[1])
    assert (c[:, :, 40:43] == 7).all()
    wide = fused(n + 1, 6, 41)
    for k, v in ((wide[:-1, :3, :40], wide[1:, :3, :40]), (wide[:-1, :3, :40], wide[:-1, :3, 1:]), (wide[:-1, :3, :40], wide[:-1, 2:5, :40]),
                 (wide[:-1, :3, :40], wide.view(-1)[:n * 3 * 40].view(n, 3, 40))):
        with pytest.raises(hq.HqmqError):
            hq.hqmq_cache4_read(w.params, w.cache, w.batch(lengths, lengths), k, v)
    assert (wide == 7).all()


def test_an_error_that_another_call_left():
    """A failed HIP call before ours is not reported as ours."""
    from paper_2605_27646_amd import binding
    hip = binding._load()  # its own dependencies' names resolve through it
    w = World(78, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 2, 40)
    w.fill_random([600, 500], F16)
    batch, k, v, q = w.batch([600, 500], [1, 1]), w.values(2, F16), w.values(2, F16), w.values(2, F16)
    out, ws = torch.empty_like(q), torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    calls = [lambda: hq.hqmq_cache4_write(w.params, w.cache, batch, k, v), lambda: hq.hqmq_cache4_read(w.params, w.cache, batch, k, v),
             lambda: hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws)]
    for call in calls:
        assert hip.hipSetDevice(1 << 20) != 0
        try:
            call()
        finally:
            hip.hipGetLastError()  # the next library's call is not to see it either
    torch.cuda.synchronize()


def test_offsets_past_32_bits():
    """Pages behind 4 GiB of codes."""
    n_pages, page, H, D = 140000, 64, 8, 128
    params = hq.Cache4Params(n_pages, page, H, D, hq.HQMQ_CACHE4_FLOAT)
    assert hq.hqmq_cache4_sizes(params)[0] > 4 << 30
    cache = hq.alloc_cache4(params, DEV)
    small = World(71, hq.HQMQ_CACHE4_FLOAT, H, D, page, 2, 2, spare=0)
    lengths = [100, 128]
    k, v = (small.values(sum(lengths), F16) for _ in range(2))
    far = np.array([[n_pages - 1, 3], [131072, n_pages - 2]], np.int32)
    tensors = (torch.tensor(lengths, dtype=torch.int32, device=DEV), torch.tensor([0, 100, 228], dtype=torch.int32, device=DEV))
    batch = hq.Cache4Batch(torch.tensor(far, device=DEV), *tensors)
    hq.hqmq_cache4_write(params, cache, batch, k, v)
    hq.hqmq_cache4_write(small.params, small.cache, small.batch(lengths, lengths), k, v)
    q = small.values(2, F16, 1.5, heads=4 * H)
    outs = []
    for p, c, b in ((params, cache, hq.Cache4Batch(torch.tensor(far, device=DEV), tensors[0])), (small.params, small.cache, small.batch(lengths))):
        out = torch.empty_like(q)
        ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(p, b, 2, 4 * H), dtype=torch.uint8, device=DEV)
        hq.hqmq_cache4_attend(p, c, b, q, 0.1, out, ws)
        outs.append(out)
    assert torch.equal(*outs)
    back = [torch.empty_like(k) for _ in range(4)]
    hq.hqmq_cache4_read(params, cache, batch, *back[:2])
    hq.hqmq_cache4_read(small.params, small.cache, small.batch(lengths, lengths), *back[2:])
    assert torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])


def test_captured_steps():
    """One captured generation step (write, attend) replayed as the lengths grow in place, against the eager calls on a second
    cache, with eager work between the replays."""
    worlds = [World(81, hq.HQMQ_CACHE4_FLOAT, 2, 128, 16, 2, 70) for _ in range(2)]
    lengths0, G = [1000, 40], 4
    for w in worlds:
        w.fill_random(lengths0, F16)
    a, b = worlds
    lengths = torch.tensor(lengths0, dtype=torch.int32, device=DEV)
    table = torch.tensor(a.table, device=DEV)
    batch = hq.Cache4Batch(table, lengths, max_length=1120)
    n_bytes = hq.hqmq_cache4_attend_workspace_bytes(a.params, batch, 2, 2 * G)
    assert n_bytes > 0
    ws, ws_eager = (torch.empty(n_bytes, dtype=torch.uint8, device=DEV) for _ in range(2))
    k, v = a.values(2, F16), a.values(2, F16)
    q = a.values(2, F16, heads=2 * G)
    out, lse = torch.empty_like(q), torch.empty(2, 2 * G, device=DEV)

    def step(w, out, lse, ws):
        hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws, lse=lse)

    lengths += 1
    step(a, out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, out, lse, ws)
    lengths -= 1
    for i in range(20):
        lengths += 1
        for x in (k, v, q):
            x.normal_()
        ws.fill_(0xFF)
        graph.replay()
        want, want_lse = torch.empty_like(q), torch.empty_like(lse)
        step(b, want, want_lse, ws_eager)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), i
    for x, y in zip(a.buffers, b.buffers):
        assert torch.equal(x, y)


def test_two_streams_at_once():
    """Calls on two streams with a workspace each give what they give one after the other; the same call twice gives the same bits."""
    w = World(91, hq.HQMQ_CACHE4_INT, 2, 96, 16, 2, 100)
    lengths = [1600, 900]
    w.fill_random(lengths, F16)
    batch = w.batch(lengths)
    n_bytes = hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, 2, 8)
    qs = [w.values(2, F16, heads=8) for _ in range(2)]

    def call(q, ws, stream=None):
        out = torch.empty_like(q)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws, stream=stream)
        return out

    wss = [torch.empty(n_bytes, dtype=torch.uint8, device=DEV) for _ in range(2)]
    want = [call(q, wss[0]) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[call(q, ws, s) for _ in range(20)] for q, ws, s in zip(qs, wss, streams)]
    torch.cuda.synchronize()
    for results, expected in zip(got, want):
        assert all(torch.equal(r, expected) for r in results)


def test_result_over_the_queries():
    w = World(95, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 2, 20)
    lengths = [300, 120]
    w.fill_random(lengths, F16)
    for rows in ([1, 1], [100, 60]):
        batch = w.batch(lengths, rows)
        q = w.values(sum(rows), F16, heads=4)
        ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, sum(rows), 4) + 1, dtype=torch.uint8, device=DEV)
        out = torch.empty_like(q)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, q, ws)
        assert torch.equal(q, out)


def test_result_beside_the_queries():
    """In the place of a fused projection's other heads, whose strides the queries have; one row of any strides over itself."""
    w = World(96, hq.HQMQ_CACHE4_FLOAT, 2, 64, 16, 2, 20)
    lengths = [300, 120]
    w.fill_random(lengths, F16)
    fused = w.values(2, F16, heads=12)
    q, out = fused[:, 4:8], torch.empty(2, 4, 64, dtype=F16, device=DEV)
    others = fused[:, :4].clone(), q.clone()
    ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(w.params, w.batch(lengths), 2, 4) + 1, dtype=torch.uint8, device=DEV)
    hq.hqmq_cache4_attend(w.params, w.cache, w.batch(lengths), q, 0.1, out, ws)
    hq.hqmq_cache4_attend(w.params, w.cache, w.batch(lengths), q, 0.1, fused[:, 8:], ws)
    assert torch.equal(fused[:, 8:], out) and torch.equal(fused[:, :4], others[0]) and torch.equal(q, others[1])
    for bad in (fused[:, 5:9], fused[:, 2:6]):
        with pytest.raises(hq.HqmqError):
            hq.hqmq_cache4_attend(w.params, w.cache, w.batch(lengths), q, 0.1, bad, ws)
    assert torch.equal(fused[:, 8:], out) and torch.equal(fused[:, :4], others[0]) and torch.equal(q, others[1])
    w.table, w.n_seqs = w.table[:1], 1
    one, single = q[:1].as_strided((1, 4, 64), (64, 768 // 12, 1)), out[:1]
    hq.hqmq_cache4_attend(w.params, w.cache, w.batch(lengths[:1]), one, 0.1, one.as_strided((1, 4, 64), (999, 64, 1)), ws)
    assert torch.equal(one, single)


def test_rows_of_no_sequence_are_left():
    """Rows before the first and behind the last sequence, with and without splits of the tokens."""
    w = World(97, hq.HQMQ_CACHE4_FLOAT, 1, 64, 16, 2, 100)
    w.fill_random([1600, 30], F16)
    table = torch.tensor(w.table, device=DEV)
    for lengths in ([1600, 30], [40, 30]):
        starts = torch.tensor([2, 3, 5], dtype=torch.int32, device=DEV)
        batch = hq.Cache4Batch(table, torch.tensor(lengths, dtype=torch.int32, device=DEV), starts, max_rows=2, max_length=max(lengths))
        q = w.values(8, F16, heads=2)
        out, lse = torch.full_like(q, 7.0), torch.full((8, 2), 7.0, device=DEV)
        ws = torch.full((hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, 8, 2) + 1,), 255, dtype=torch.uint8, device=DEV)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws, lse=lse)
        torch.cuda.synchronize()
        outside = [0, 1, 5, 6, 7]
        assert (out[outside] == 7).all() and (lse[outside] == 7).all() and not (out[2:5] == 7).all()


def test_no_allocation_by_the_calls():
    w = World(99, hq.HQMQ_CACHE4_FLOAT, 2, 128, 16, 1, 100)
    w.fill_random([1500], F16)
    batch = w.batch([1500])
    q = w.values(1, F16, heads=8)
    k, v, out = w.values(1, F16), w.values(1, F16), torch.empty_like(q)
    ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, 1, 8), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    hq.hqmq_cache4_write(w.params, w.cache, batch, k, v)
    hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.1, out, ws)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
