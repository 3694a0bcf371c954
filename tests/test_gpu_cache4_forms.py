"""Attention over the paged 4-bit cache by workgroups of 32 and 64 query rows: every form of the kernel that has them, asked of the library's
own plan, against the plain numpy form (cache4_ref.py) with the bounds that it adds up."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import cache4_ref as ref
import paper_2605_27646_amd as hq
from cache4_plan import plan
from test_gpu_cache4 import BF16, DEV, F16, FMT, HALF, WEIGHT, World, _check_attend, _np

pytestmark = pytest.mark.gpu


def _plan(w, rows, G, **hints):
    return plan(w.H, w.D, w.page, w.n_seqs, w.table.shape[1], int(sum(rows)), w.H * G, **hints)


def _world(seed, fmt, D, blocks, page=16):
    """Sequences enough for workgroups of `blocks` x 16 rows, none with a multiple of them, some with less than one: (world, lengths, rows, G).
    4 waves take 128 tokens a round: lengths end in every wave, in the first round and the third."""
    if blocks == 2:
        w, rows, G = World(seed, fmt, 8, D, page, 12, 20), [12, 11, 14, 11, 12, 13, 4, 11, 16, 11, 12, 11], 3
    else:
        w, rows, G = World(seed, fmt, 16, D, page, 12, 20), [13, 14, 13, 15, 13, 26, 13, 5, 13, 16, 13, 13], 5
    return w, [300, 33, 129, 64, 97, 31, 8, 200, 16, 77, 48, 160], rows, G


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,blocks", [(32, 2), (64, 2), (96, 2), (128, 2), (192, 2), (256, 2), (32, 4), (64, 4), (96, 4), (128, 4)])
def test_every_form(fmt, dtype, D, blocks):
    w, lengths, rows, G = _world(D + blocks, fmt, D, blocks)
    w.fill_random(lengths, dtype, hot=True)
    for flat, hints in ((False, dict(max_rows=max(rows))), (True, {})):  # a place for each tile of the largest sequence, or along all rows
        p = _plan(w, rows, G, **hints)
        assert p.blocks == blocks and p.flat == flat and p.n_splits == 1
        _check_attend(w, lengths, rows, dtype, G, **hints)


@pytest.mark.parametrize("blocks", [2, 4])
@pytest.mark.parametrize("window", [1, 20, 70])
@pytest.mark.parametrize("fmt,dtype", [(FMT[0], BF16), (FMT[1], F16)])
def test_windows(fmt, dtype, window, blocks):
    """Pages before the sequences' windows are none, or another's with NaN scales."""
    w, lengths, rows, G = _world(window, fmt, 64, blocks)
    assert _plan(w, rows, G, window=window).blocks == blocks
    w.fill_random(lengths, dtype)
    other = [p for p in range(w.params.n_pages) if p not in set(w.table.ravel())][0]  # never written
    for i, length in enumerate(lengths):
        given_back = max(0, length - rows[i] + 1 - window) // 16
        w.table[i, :given_back:2], w.table[i, 1:given_back:2] = other, -1
        w.table[i, -(-length // 16):] = other
    _check_attend(w, lengths, rows, dtype, G, window=window)


@pytest.mark.parametrize("D,blocks", [(17, 2), (100, 2), (130, 2), (251, 2), (5, 4), (60, 4), (90, 4), (125, 4)])
@pytest.mark.parametrize("fmt,dtype", [(FMT[0], F16), (FMT[1], BF16)])
def test_odd_heads_and_strides(fmt, dtype, D, blocks):
    w, lengths, rows, G = _world(D, fmt, D, blocks)
    assert _plan(w, rows, G).blocks == blocks
    w.fill_random(lengths, dtype)
    _check_attend(w, lengths, rows, dtype, G, strided=True)


@pytest.mark.parametrize("fmt,dtype", [(FMT[0], F16), (FMT[1], BF16)])
@pytest.mark.parametrize("blocks", [2, 4])
@pytest.mark.parametrize("scale", [-0.3, 4.0])
def test_tokens_without_a_place(fmt, dtype, blocks, scale):
    """Pages that are none inside the sequences, more rows than tokens, lengths of nothing; negative scales, and scores of which one takes all."""
    w, lengths, rows, G = _world(blocks, fmt, 96, blocks)
    w.fill_random(lengths, dtype)
    w.table[0, 1], w.table[2, 0], w.table[3, 2], w.table[7, 5:9] = -1, w.params.n_pages, 2 ** 31 - 1, -5
    lengths[5], lengths[8] = 0, 3
    assert _plan(w, rows, G).blocks == blocks
    _check_attend(w, lengths, rows, dtype, G, scale=scale)


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("blocks", [2, 4])
def test_queries_that_are_not_finite(fmt, dtype, blocks):
    """They give NaN where they see a token and nothing to the other rows of their workgroup."""
    w, lengths, rows, G = _world(7, fmt, 64, blocks)
    w.fill_random(lengths, dtype)
    lengths[3] = 0  # its rows see none
    assert _plan(w, rows, G).blocks == blocks
    n, Hq = sum(rows), w.H * G
    q, batch = w.values(n, dtype, heads=Hq), w.batch(lengths, rows)
    ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, n, Hq) + 1, dtype=torch.uint8, device=DEV)
    results = []
    lost = torch.zeros(n, Hq, dtype=torch.bool)
    for turn in range(2):
        out, lse = torch.empty_like(q), torch.empty(n, Hq, device=DEV)
        hq.hqmq_cache4_attend(w.params, w.cache, batch, q, 0.125, out, ws, lse=lse)
        results.append((out.cpu(), lse.cpu()))
        if turn == 0:
            for row in range(0, n, 2):
                head = 5 * row % Hq
                q[row, head, 7 * row % 64] = [float("nan"), float("inf"), -float("inf")][row % 3]
                lost[row, head] = True
    (a, la), (b, lb) = results
    pos = np.array([p for _, _, p in w.places(lengths, rows)])
    empty = torch.tensor(pos < 0)[:, None].expand(-1, Hq)
    assert torch.equal(a[~lost], b[~lost]) and torch.equal(la[~lost], lb[~lost])
    assert b[lost & ~empty].isnan().all() and lb[lost & ~empty].isnan().all() and (lost & ~empty).any()
    assert (b[empty] == 0).all() and (lb[empty] == -float("inf")).all() and (lost & empty).any()


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype,size", [(F16, 60000.0), (BF16, 2.0 ** 90)])
@pytest.mark.parametrize("blocks", [2, 4])
def test_scores_of_any_size(fmt, dtype, size, blocks):
    """Rows whose scores pass 2^27, all their weight on one token or shared by two that tie, beside rows of ordinary scores in one workgroup."""
    w, lengths, rows, G = _world(9, fmt, 64, blocks)
    n, scale = sum(lengths), 1024.0
    assert _plan(w, rows, G).blocks == blocks
    k, v = w.values(n, dtype), w.values(n, dtype)
    first = np.concatenate([[0], np.cumsum(lengths)])
    k[:, :, 0] = 2.0
    for i, length in enumerate(lengths):
        k[first[i], :, 0] = 4.0  # the first token of each, and another where every row sees it
        if i % 2 and length > rows[i] + 2:
            k[first[i] + length - rows[i] - 1, :, 0] = 4.0
    hq.hqmq_cache4_write(w.params, w.cache, w.batch(lengths, lengths), k, v)
    w.write_plain(lengths, lengths, k, v)
    q = w.values(sum(rows), dtype, heads=w.H * G) / 4096
    far = torch.arange(sum(rows) * w.H * G, device=DEV).view(sum(rows), -1) % 3 == 0
    q[far] = 0
    q[:, :, 0] = torch.where(far, size, q[:, :, 0])
    out, lse = torch.full_like(q, float("nan")), torch.empty(q.shape[:2], device=DEV)
    batch = w.batch(lengths, rows)
    ws = torch.empty(hq.hqmq_cache4_attend_workspace_bytes(w.params, batch, sum(rows), w.H * G) + 1, dtype=torch.uint8, device=DEV)
    hq.hqmq_cache4_attend(w.params, w.cache, batch, q, scale, out, ws, lse=lse)
    got, got_lse, qn, far = _np(out), _np(lse), _np(q), far.cpu().numpy()
    near_rows = np.zeros(w.n_seqs, int)
    for row, i, pos in w.places(lengths, rows):
        if pos < 0:
            assert (got[row] == 0).all()
            continue
        near_rows[i] += 1
        kk, there = w.plain.sequence(0, w.table[i], lengths[i]) if near_rows[i] == 1 else (kk, there)
        vv = w.plain.sequence(1, w.table[i], lengths[i])[0] if near_rows[i] == 1 else vv
        if near_rows[i] == 1 or row % 4 == 0:  # the ordinary ones: some are enough
            some = [h for h in range(w.H * G) if not far[row, h]]
            o, l, tol, tol_l = ref.attend(qn[row][None], kk, vv, there, np.array([pos]), scale, 0, HALF[dtype], WEIGHT[dtype])
            assert (np.abs(got[row] - o[0])[some] <= tol[0][some]).all() and (np.abs(got_lse[row] - l[0])[some] <= tol_l[0][some]).all()
        for head in range(w.H * G):
            if not far[row, head]:
                continue
            x = kk[:pos + 1, head // G, 0]
            tokens = np.flatnonzero(x == x.max())
            others = x[x < x.max()]
            s = scale * float(q[row, head, 0]) * x.max()
            if len(others):  # a step of the codes at least between them, which is far more than 200
                assert s - scale * float(q[row, head, 0]) * others.max() > 200
            want = vv[tokens, head // G].mean(0)
            size_of = np.abs(vv[tokens, head // G]).mean(0)
            # ties weigh the same to 2^-11 of a weight or nothing, each sum over n tokens is off by n 2^-23 and the rest by 2^-20
            assert (np.abs(got[row, head] - want) <= HALF[dtype] * np.abs(want) + (2.0 ** -20 + len(tokens) * 2.0 ** -23) * size_of + 2.0 ** -25).all(), (row, head)
            assert abs(got_lse[row, head] - s) <= abs(s) * 2.0 ** -21 + 1


@pytest.mark.parametrize("fmt", FMT)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128, 200])
def test_split_tokens(fmt, dtype, D):
    """32 rows of a workgroup and the tokens in parts."""
    w = World(D, fmt, 8, D, 32, 1, 36)
    rows, G = [67], 8
    p = _plan(w, rows, G, max_length=1100)
    assert p.blocks == 2 and p.n_splits > 1 and not p.flat
    w.fill_random([1100], dtype)
    _check_attend(w, [1100], rows, dtype, G, max_length=1100)


@pytest.mark.parametrize("fmt,dtype", [(FMT[0], F16), (FMT[1], BF16)])
@pytest.mark.parametrize("H,n,blocks,length", [(8, 70, 4, 220), (2, 90, 2, 220), (2, 90, 2, 700)])
def test_places_along_all_rows(fmt, dtype, H, n, blocks, length):
    """One sequence with most rows, dealt along all of them, with the tokens in parts where they are many."""
    w = World(H + n, fmt, H, 64, 32, n, length // 32 + 1)
    rows = [1] * n
    rows[0], rows[13], rows[40], rows[n - 1] = 0, 203, 11, 0
    lengths = [int(x) for x in w.rng.integers(1, 60, n)]
    lengths[13], lengths[50] = 215, length
    p = _plan(w, rows, 4, max_rows=203, max_length=length)
    assert p.blocks == blocks and p.flat and (p.n_splits > 1) == (length > 512)
    w.fill_random(lengths, dtype)
    _check_attend(w, lengths, rows, dtype, 4, max_rows=203, max_length=length)
