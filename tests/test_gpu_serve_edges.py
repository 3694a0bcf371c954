"""Edges of the calls that serve a batch from packed caches, beside test_gpu_serve.py and with its helpers: keys that are not
finite, limits far outside, weights' bits, and the forms of each kernel."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2605_27646_amd as hq
from gpu_util import gpu_encode
import test_gpu_serve as serve
from test_gpu_serve import DEV, Cache, _gen, _secs

pytestmark = pytest.mark.gpu


def _put_payloads(cache, first, end, values):
    """The payloads of every (b, h)'s tokens first .. end - 1 become `values`; returns which tokens have any."""
    off = cache.bufs.row_off.cpu().numpy().view(np.uint32)
    pay = cache.bufs.outliers.cpu().numpy().copy()
    has = np.zeros((cache.B, cache.H, cache.T), bool)
    for b in range(cache.B):
        for h in range(cache.H):
            r0 = (b * cache.H + h) * cache.T
            pay.reshape(-1, 4)[off[r0 + first]:off[r0 + end]] = values
            has[b, h, first:end] = np.diff(off[r0 + first:r0 + end + 1].astype(np.int64)) > 0
    assert has.any()
    cache.bufs.outliers.copy_(torch.from_numpy(pay))
    return torch.from_numpy(has)


# ---- accumulated weight --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("M,G", [(1, 1), (1, 2), (1, 4), (3, 4), (1, 16), (16, 4), (33, 4), (130, 1), (65, 4)])
@pytest.mark.parametrize("D", [128, 64])
def test_mass_of_keys_that_nobody_sees(M, G, D):
    """A padded batch: infinities and NaN in keys behind every limit change no bit, and add nothing to their own tokens."""
    B, H, T, most = 2, 2, 333, 217
    sec, _ = _secs(13, H, 64)
    k = Cache(1400 + D, B, H, T, D, sec, Cmul=1.2)
    N = B * M
    q = torch.randn(N, H * G, D, generator=_gen(1420)).to(torch.float16).to(DEV)
    lse = (torch.randn(N, H * G, generator=_gen(1421)) + 6.0).to(DEV)
    visible = torch.full((N, H * G), most, dtype=torch.int32, device=DEV)
    mass = torch.rand(B, H, T, generator=_gen(1422)).to(DEV)

    def run():
        out = torch.full_like(mass, float("nan"))
        hq.hqmq_attend_mass(k.params, q, D ** -0.5, k.bufs, k.sec, lse, mass, decay=0.5, visible=visible, out=out)
        return out.cpu()

    clean = run()
    _put_payloads(k, most, T, [np.nan, np.inf, -np.inf, 1.0])
    got = run()
    assert torch.equal(got[..., most:], 0.5 * mass[..., most:].cpu())
    assert torch.equal(got, clean)


@pytest.mark.parametrize("M,G", [(1, 1), (1, 4), (3, 4), (16, 4), (33, 4)])
def test_mass_of_infinite_keys(M, G):
    """Keys whose every score is minus infinity weigh nothing, where no limits are given too; a query head that saw nothing (an
    lse of minus infinity) adds nothing, also where its score is plus infinity."""
    B, H, T, D = 1, 2, 333, 64
    sec, _ = _secs(13, H, 64)
    k = Cache(1500, B, H, T, D, sec, Cmul=1.2)
    q = torch.rand(M, H * G, D, generator=_gen(1520)) + 0.5
    lse = torch.full((M, H * G), 9.0)
    if M * G > 1:
        q[0, ::G] *= -1.0  # the first query head of every kv head
        lse[0, ::G] = float("-inf")
    q, lse = q.to(torch.float16).to(DEV), lse.to(DEV)
    has = _put_payloads(k, 100, 200, [-np.inf, -1.0, -1.0, -np.inf])
    mass = torch.rand(B, H, T, generator=_gen(1522)).to(DEV)
    out = torch.full_like(mass, float("nan"))
    hq.hqmq_attend_mass(k.params, q, D ** -0.5, k.bufs, k.sec, lse, mass, out=out)
    out, mass = out.cpu(), mass.cpu()
    assert torch.isfinite(out).all()
    assert torch.equal(out[has], mass[has])
    assert (out[~has] > mass[~has]).any()


# ---- limits --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,S,flags", [(1, 16, 0), (5, 16, 0), (130, 300, 0), (3000, 16, 0), (3000, 300, 0), (3000, 64, hq.HQMQ_FLAG_ATTEND_TABLES)])
@pytest.mark.parametrize("G", [16, 3])
def test_attention_with_limits_far_below_zero(T, S, flags, G):
    """The lowest limits there are mean that nothing is seen: by every query head, and by some beside others that see all."""
    B, H, D, low = 2, 2, 128, -(2 ** 31)
    sk, sv = _secs(17, H, S)
    k, v = Cache(1700, B, H, T, D, sk), Cache(1701, B, H, T, D, sv)
    p = hq.HqmqParams(B, H, T, D, H * T * D, T * D, D, S, k.b_r, 3.0, flags)
    q = torch.randn(B, H * G, D, generator=_gen(1702)).to(torch.float16).to(DEV)
    ws = torch.empty(hq.hqmq_attend_workspace_bytes(p, H * G), dtype=torch.uint8, device=DEV)

    def run(visible):
        out, lse = torch.full_like(q, float("nan")), torch.full((B, H * G), float("nan"), device=DEV)
        hq.hqmq_attend_masked(p, q, 0.09, k.bufs, k.sec, v.bufs, v.sec, visible.to(DEV), out, ws, lse)
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    none = torch.full((B, H * G), low, dtype=torch.int32)
    out, lse = run(none)
    assert not out.any() and torch.isneginf(lse).all()
    some = torch.full((B, H * G), T, dtype=torch.int32)
    whole = run(some)
    some[:, ::2] = low
    some[0, 0] = -T
    out, lse = run(some)
    blind = some < 0
    assert not out[blind].any() and torch.isneginf(lse[blind]).all()
    assert torch.equal(out[~blind], whole[0][~blind]) and torch.equal(lse[~blind], whole[1][~blind])


@pytest.mark.parametrize("M,G,T,own", [(2, 16, 40, 200), (9, 16, 40, 300), (40, 2, 40, 70), (20, 16, 70, 1)])
def test_shared_with_limits_far_below_zero(M, G, T, own):
    """The same for prefix and own tokens, own tokens in the prefix's launch and in one of their own."""
    H, D, S, low = 2, 64, 24, -(2 ** 31)
    sk, sv = _secs(19, H, S)
    k, v = Cache(1900, 1, H, T, D, sk), Cache(1901, 1, H, T, D, sv)
    ok, ov = Cache(1902, M, H, own, D, sk), Cache(1903, M, H, own, D, sv)
    q = torch.randn(M, H * G, D, generator=_gen(1904)).to(torch.float16).to(DEV)
    ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(k.params, M, H * G, ok.params), dtype=torch.uint8, device=DEV)

    def run(limit, own_limit):
        out, lse = torch.full_like(q, float("nan")), torch.full((M, H * G), float("nan"), device=DEV)
        visible, own_visible = (torch.full((M, H * G), x, dtype=torch.int32, device=DEV) for x in (limit, own_limit))
        hq.hqmq_attend_shared(k.params, q, 0.1, k.bufs, k.sec, v.bufs, v.sec, out, ws, lse=lse, visible=visible,
                              own=hq.OwnTokens(ok.params, ok.bufs, ov.bufs, own_visible))
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    out, lse = run(low, low)
    assert not out.any() and torch.isneginf(lse).all()
    for got, want in ((run(T, low), run(T, 0)), (run(low, own), run(0, own))):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- weights' bits -------------------------------------------------------------------------------------------------

def _verbatim(x, sec):
    """Packed rows whose chunks are zeros or kept as they are: at most every fourth chunk of x is not zero, so that the median
    norm is zero and every other chunk lies above it."""
    g = gpu_encode(x.to(torch.float16).to(DEV), sec, 6, 3.0)
    back = torch.empty(x.shape, dtype=torch.float16, device=DEV)
    hq.hqmq_decode(g.params, g.bufs, sec, back)
    assert torch.equal(back.cpu(), x.to(torch.float16))
    return g


@pytest.mark.parametrize("M", [10, 20, 33])
@pytest.mark.parametrize("D", [128, 96, 64])
@pytest.mark.parametrize("rise", [16.5, 20.5, 24.5, 25.5, 26.5, 30.5])
def test_shared_weights_far_below_a_later_one(M, D, rise):
    """Scores 0 of 32 tokens, 4.9 of the next 32, then one of `rise` and some far below, in the log2 domain: the middle ones' weights are down to
    2^-26 of the last one's, and their values as much larger.  One value per token and query row counts, so that the result is the
    weighted sum of the middle tokens' values.  A weight is off by 2^-22 of itself or 2^-34 of the largest one (fp16 pairs); arithmetic
    and exponents 1e-4, the result 2^-11."""
    B, H, G, T, S = 1, 256, 4, 96, 16
    sec = torch.stack([_secs(23, 1, S)[0][0]] * H).to(DEV)
    s2 = torch.full((T,), -90.0)
    s2[:32], s2[32:64], s2[64] = 0.0, 4.9, rise
    k, v = torch.zeros(B, H, T, D), torch.zeros(B, H, T, D)
    k[..., 0] = s2.to(torch.float16)
    v[:, :, 32:64, :8] = 6e4 * (0.5 + 0.5 * torch.rand(B, H, 32, 8, generator=_gen(2300)))
    gk, gv = _verbatim(k, sec), _verbatim(v, sec)
    q = torch.zeros(M, H * G, D, dtype=torch.float16)
    q[..., 0] = 1.0
    scale = math.log(2.0)
    out, lse = torch.full((M, H * G, D), float("nan"), dtype=torch.float16, device=DEV), torch.empty(M, H * G, device=DEV)
    ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(gk.params, M, H * G), dtype=torch.uint8, device=DEV)
    hq.hqmq_attend_shared(gk.params, q.to(DEV), scale, gk.bufs, sec, gv.bufs, sec, out, ws, lse=lse)
    torch.cuda.synchronize()
    w = torch.exp2(k[0, 0, :, 0].to(torch.float16).double() - rise)
    v64 = v[0].to(torch.float16).double()
    want = (w[:, None] * v64).sum(1) / w.sum()  # [H, D]
    bound = (2.0 ** -11 + 1e-4) * want + 2.0 ** -34 * v64.sum(1) + 2.0 ** -24
    got = out.cpu().double().view(M, H, G, D)
    err = (got - want[None, :, None]).abs()
    assert (want[:, :8] > 0.02).all()
    assert (err <= bound[None, :, None]).all(), (err.max().item(), want.max().item(), got.max().item())


def _check_by_sixty_four(got, lse, q, scale, K, V, visible, own_kv, own_visible, B, M, H, G):
    """test_gpu_serve._check_shared with its bound for up to 64 query rows of a kv head, whatever their number: 1e-4 of the weighted sum of
    |V|, of which weights of 22 bits take 2^-22."""
    class Some:
        def __init__(self, c, first, end):
            self.hat, self.slack = c.hat[first:end], c.slack[first:end]

    step = 64 // G
    for b in range(B):
        for first in range(b * M, (b + 1) * M, step):
            seq = slice(first, min(first + step, (b + 1) * M))
            cut = lambda x: None if x is None else x[seq]  # noqa: E731
            of_seq = None if own_kv is None else tuple(Some(c, seq.start, seq.stop) for c in own_kv)
            serve_check(got[seq], lse[seq], q[seq], scale, Some(K, b, b + 1), Some(V, b, b + 1), cut(visible), of_seq, cut(own_visible), 1,
                        seq.stop - seq.start, H, G)


serve_check = serve._check_shared


@pytest.fixture
def tight(monkeypatch):
    """serve._shared, its outputs held to 22-bit weights at every number of query rows."""
    monkeypatch.setattr(serve, "_check_shared", _check_by_sixty_four)
    return serve._shared


@pytest.mark.parametrize("M,G,own", [(17, 4, 0), (32, 4, 30), (9, 11, 0), (33, 4, 0), (64, 4, 30), (65, 4, 0), (20, 16, 7)])
@pytest.mark.parametrize("D", [128, 96, 64])
@pytest.mark.parametrize("gain", [30.0, 2.0])
def test_shared_weights_of_many_rows(tight, M, G, own, D, gain):
    """One token with nearly all of the weight, and many: no query row's weights have fewer bits for there being more rows."""
    tight(2500 + M + D, 1, M, 2, G, 333, D, 24, own=own, gain=gain)


# ---- many rows -----------------------------------------------------------------------------------------------------

def test_windows_of_many_positions(tight):
    """The last 1024 positions of two prompts: four workgroups' rows of each kv head, 65536 query heads in all."""
    tight(2700, 2, 1024, 32, 1, 40, 64, 16, limits="ragged")
    tight(2710, 1, 1024, 2, 2, 70, 128, 16)
    serve._mass(2720, 2, 1024, 32, 1, 40, 64, 16, limits="ragged")


# ---- every form of the attention -----------------------------------------------------------------------------------

def _shares(B, M, H, G, T, D, S):
    """Workgroups along the prefix that the call plans: its workspace has 130 floats for each of them and query head."""
    p = hq.HqmqParams(B, H, T, D, H * T * D, T * D, D, S, 6, 3.0, 0)
    return hq.hqmq_attend_shared_workspace_bytes(p, M, H * G) // (B * M * H * G * 520)


@pytest.mark.parametrize("M,G", [(3, 4), (25, 4), (35, 4), (65, 4)])
@pytest.mark.parametrize("D", [128, 96, 64])
@pytest.mark.parametrize("S", [5, 512, 700, 1024, 2730])
def test_shared_codebooks_of_every_form(tight, M, G, D, S):
    """Up to 64, 128, 256 query rows and more, of powers of two and others, with tables of directions and without (from 600 secondaries
    on, more than 128 rows from 900)."""
    tight(2800 + M + D + S, 1, M, 1, G, 170, D, S, 4 if S == 5 else 6)


@pytest.mark.parametrize("M", [30, 40])
@pytest.mark.parametrize("D", [128, 96, 64])
@pytest.mark.parametrize("Cmul,capacity,kgain,gain", [
    (0.3, None, 1.0, 1.0), (1.2, 37, 1.0, 1.0), (3.0, 0, 1.0, 1.0), (3.0, None, 9000.0, 1e-3), (3.0, None, 1e-4, 3.0),
])
def test_shared_outliers_and_ranges_of_many_rows(tight, M, D, Cmul, capacity, kgain, gain):
    """The careful form beside more than 64 and 128 rows: saturating scales, payloads past the staged ones, lists too short."""
    tight(2900 + M + D, 1, M, 2, 4, 321, D, 64, 6, Cmul=Cmul, capacity=capacity, kgain=kgain, gain=gain)


@pytest.mark.parametrize("B,M,G,D,T,Cmul,limits", [
    (64, 35, 4, 128, 333, 3.0, None), (64, 35, 4, 128, 257, 0.5, "ragged"), (64, 33, 4, 96, 333, 3.0, "some"), (64, 40, 4, 64, 500, 1.2, "ragged"),
    (128, 25, 4, 128, 333, 1.2, "ragged"), (192, 3, 4, 128, 333, 1.2, "ragged"), (32, 70, 4, 128, 130, 1.2, "ragged"),
])
def test_shared_many_tiles_of_one_workgroup(tight, B, M, G, D, T, Cmul, limits):
    """As many heads as the chip takes at once: a workgroup goes through all of its head's tiles."""
    H = 4
    assert _shares(B, M, H, G, T, D, 24) == 1
    tight(3000 + M + D, B, M, H, G, T, D, 24, 6, limits=limits, Cmul=Cmul)


@pytest.mark.parametrize("M,G,D,own", [(3, 4, 128, 20), (25, 4, 96, 200), (35, 4, 64, 90), (40, 8, 128, 300)])
def test_shared_negative_scale(M, G, D, own):
    """The scores of the negated queries: of the prefix to the bit, as its kernel takes the sign into the queries; hqmq_attend's, which own
    tokens may take, into the product, whose fp32 sums need not round alike for both signs."""
    H, T, S = 2, 270, 24
    sk, sv = _secs(29, H, S)
    k, v = Cache(3100, 1, H, T, D, sk), Cache(3101, 1, H, T, D, sv)
    ok, ov = Cache(3102, M, H, own, D, sk), Cache(3103, M, H, own, D, sv)
    q = torch.randn(M, H * G, D, generator=_gen(3104)).to(torch.float16)
    ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(k.params, M, H * G, ok.params), dtype=torch.uint8, device=DEV)
    tokens = hq.OwnTokens(ok.params, ok.bufs, ov.bufs)

    def run(q, scale, tokens):
        out, lse = torch.full(q.shape, float("nan"), dtype=torch.float16, device=DEV), torch.full((M, H * G), float("nan"), device=DEV)
        hq.hqmq_attend_shared(k.params, q.to(DEV), scale, k.bufs, k.sec, v.bufs, v.sec, out, ws, own=tokens, lse=lse)
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    got, want = run(q, -0.11, None), run(-q, 0.11, None)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    got = run(q, -0.11, tokens)
    _check_by_sixty_four(got[0].numpy(), got[1].numpy().astype(np.float64), -q.numpy(), float(np.float32(0.11)), k.decoded(), v.decoded(), None,
                         (ok.decoded(), ov.decoded()), None, 1, M, H, G)


@pytest.mark.parametrize("B,M,H,G,D,T", [(140, 9, 6, 3, 128, 71), (129, 9, 6, 3, 96, 71), (65, 25, 8, 4, 64, 130), (66, 40, 4, 4, 128, 40), (1, 3, 2, 4, 64, 128)])
@pytest.mark.parametrize("limits", [None, "some"])
def test_shared_results_of_one_share(tight, B, M, H, G, D, T, limits):
    """Where one workgroup has all of its rows' prefix it writes the result itself, without partial sums."""
    assert _shares(B, M, H, G, T, D, 16) == 1
    tight(3200 + B + M, B, M, H, G, T, D, 16, 4, limits=limits)
