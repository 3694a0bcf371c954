"""Serving a batch from packed caches on the GPU: attention over shared prefixes and own tokens, accumulated attention
weight, the choice of the tokens to keep and the compaction of packed tensors, against plain fp64 / integer references
computed from the same packed bytes (which the oracle decodes)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import oracle
import paper_2605_27646_amd as hq
from gpu_util import gpu_encode
from test_gpu_attend import Decoded

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LOG2E = 1.0 / math.log(2.0)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _secs(seed, H, S):
    cb = hq.hqmq_build_codebooks(seed, 1, H, S)
    return [cb[0, i].contiguous() for i in range(2)]


class Cache:
    """A packed K (or V) tensor and its fp16 reconstruction: hat, and slack where fp32 arithmetic may round an element to
    the neighbouring fp16 value (test_gpu_attend.Decoded)."""

    def __init__(self, seed, B, H, T, D, sec, b_r=6, Cmul=3.0, gain=1.0, capacity=None, channel=0.5):
        g = _gen(seed)
        x = torch.randn(B, H, T, D, generator=g) * torch.exp(channel * torch.randn(1, H, 1, D, generator=g)) * gain
        x = x.clamp(-65504, 65504).to(torch.float16)
        self.sec_np, self.sec = sec.numpy(), sec.to(DEV)
        self.B, self.H, self.T, self.D, self.b_r = B, H, T, D, b_r
        self.g = gpu_encode(x.to(DEV), self.sec, b_r, Cmul, outlier_capacity=capacity)
        self.params, self.bufs = self.g.params, self.g.bufs

    def decoded(self):
        return decoded_of(self.bufs, self.params, self.sec_np)


class _Bytes:
    pass


def decoded_of(bufs, p, sec_np):
    """Decoded of the bytes that the buffers hold now."""
    e = _Bytes()
    u32 = lambda t: t.cpu().numpy().view(np.uint32)  # noqa: E731
    e.codes, e.flags, e.row_off = u32(bufs.codes), u32(bufs.flags), u32(bufs.row_off)
    e.sigma = bufs.sigma.cpu().numpy().view(np.uint16)
    total, cap = int(e.row_off[-1]), bufs.outlier_capacity
    outl = np.zeros((max(total, 1), 4), np.uint16)  # a payload beyond the list decodes to zeros
    kept = min(total, cap)
    outl[:kept] = bufs.outliers[:kept].cpu().numpy().view(np.uint16).reshape(kept, 4)
    e.outliers = outl
    return Decoded(e, sec_np, p.B, p.H, p.T, p.b_r, p.D)


def _rows(x, B, M, H, G):
    """[B M, H G, ...] -> [B, H, M G, ...]"""
    return np.moveaxis(x.reshape(B, M, H, G, *x.shape[2:]), 1, 2).reshape(B, H, M * G, *x.shape[2:])


def _back(x, B, M, H, G):
    return np.moveaxis(x.reshape(B, H, M, G, *x.shape[3:]), 2, 1).reshape(B * M, H * G, *x.shape[3:])


def _scores(q, K, scale, visible, B, M, H, G):
    """fp64 scores of every query row [B, H, R, T] (-inf where not visible), what an element that may round the other way can
    move them by, and the sum of the products' magnitudes."""
    qf = _rows(q.astype(np.float64), B, M, H, G)
    s = scale * (qf @ np.swapaxes(K.hat, 2, 3))
    delta = scale * (np.abs(qf) @ np.swapaxes(K.slack, 2, 3))
    size = scale * (np.abs(qf) @ np.swapaxes(np.abs(K.hat), 2, 3))
    if visible is not None:
        v = _rows(visible, B, M, H, G)
        s = np.where(np.arange(K.hat.shape[2]) < v[..., None], s, -np.inf)
    return s, delta, size


def _check_shared(got, lse, q, scale, K, V, visible, own_kv, own_visible, B, M, H, G):
    """The bound of test_gpu_attend._check, per output element, over prefix and own tokens: 2^-11 |o| for the fp16 rounding;
    elements of V_hat and K_hat that may round the other way, weighted by what they carry; 1e-4 of the weighted sum of |V|
    for the fp32 arithmetic (22-bit weights, exp2, sums).  Where more than 64 query rows share the prefix its weights are rounded
    to fp16 once: each is off by at most 2^-11 of itself, so the sum of w_t v_t by at most 2^-11 of the weighted sum of |V|."""
    D = q.shape[2]
    weights = 1e-4 + (2.0 ** -11 if M * G > 64 else 0.0)
    parts = [(K, V, visible, B, M)]
    if own_kv is not None:
        parts.append((own_kv[0], own_kv[1], own_visible, B * M, 1))
    sc = []
    for k, v, vis, b, m in parts:
        s, delta, _ = _scores(q, k, scale, vis, b, m, H, G)
        sc.append((_back(s, b, m, H, G), _back(delta, b, m, H, G), v, b, m))
    top = np.max([s.max(-1) for s, *_ in sc], 0)
    base = np.where(np.isfinite(top), top, 0.0)
    total = sum(np.exp(s - base[..., None]).sum(-1) for s, *_ in sc)
    o, A, from_v, pd_sum, pd_v = 0.0, 0.0, 0.0, 0.0, 0.0
    for s, delta, v, b, m in sc:
        p = np.exp(s - base[..., None]) / np.where(total > 0, total, 1.0)[..., None]
        pr, pdr = _rows(p, b, m, H, G), _rows(p * delta, b, m, H, G)
        o = o + _back(pr @ v.hat, b, m, H, G)
        A = A + _back(pr @ np.abs(v.hat), b, m, H, G)
        from_v = from_v + _back(pr @ v.slack, b, m, H, G)
        pd_v = pd_v + _back(pdr @ np.abs(v.hat), b, m, H, G)
        pd_sum = pd_sum + (p * delta).sum(-1)
    bound = 2.0 ** -11 * np.abs(o) * 1.001 + from_v + 1.5 * (pd_v + np.abs(o) * pd_sum[..., None]) + weights * A + 2.0 ** -24
    err = np.abs(got.astype(np.float64) - o)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), (float(err.max()), np.argwhere(err > bound)[:5], err[err > bound][:5], bound[err > bound][:5])
    with np.errstate(divide="ignore"):
        want = base + np.log(total)
    assert np.array_equal(np.isneginf(lse), np.isneginf(want))
    fin = np.isfinite(want)
    tol = 2e-5 * np.maximum(1.0, np.abs(np.where(fin, want, 0.0))) + 1.5 * pd_sum
    assert (np.abs(lse[fin] - want[fin]) <= tol[fin]).all()
    assert (got[~fin] == 0).all()


def _limits(kind, N, heads, T, seed):
    g = _gen(seed)
    if kind is None:
        return None
    v = torch.randint(-2, T + 5, (N, heads), generator=g)
    if kind == "none":
        v = torch.zeros(N, heads, dtype=torch.int64)
    if kind == "some":  # whole sequences, and single heads, that see nothing
        v[: max(1, N // 2)] = 0
        v[-1, 0] = -3
    return v.to(torch.int32)


def _shared(seed, B, M, H, G, T, D, S, b_r=6, own=0, limits=None, own_limits=None, gain=1.0, Cmul=3.0, kgain=1.0, capacity=None,
            stream=None):
    sk, sv = _secs(seed, H, S)
    k, v = (Cache(seed + 1 + i, B, H, T, D, s, b_r, Cmul, kgain, capacity) for i, s in enumerate((sk, sv)))
    N = B * M
    q = (torch.randn(N, H * G, D, generator=_gen(seed + 3)) * gain).to(torch.float16)
    vis = _limits(limits, N, H * G, T, seed + 4)
    tokens = ok = ov = None
    own_vis = _limits(own_limits, N, H * G, own, seed + 5)
    if own:
        ok, ov = (Cache(seed + 7 + i, N, H, own, D, s, b_r, Cmul, kgain, capacity) for i, s in enumerate((sk, sv)))
        tokens = hq.OwnTokens(ok.params, ok.bufs, ov.bufs, None if own_vis is None else own_vis.to(DEV))
    ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(k.params, M, H * G, ok.params if own else None), dtype=torch.uint8, device=DEV)
    ws.fill_(0xCD)
    q_dev = q.to(DEV)
    out = torch.full_like(q_dev, float("nan"))
    lse = torch.full((N, H * G), float("nan"), device=DEV)
    scale = 1.0 / math.sqrt(D)
    hq.hqmq_attend_shared(k.params, q_dev, scale, k.bufs, k.sec, v.bufs, v.sec, out, ws, own=tokens,
                          visible=None if vis is None else vis.to(DEV), lse=lse)
    torch.cuda.synchronize()
    _check_shared(out.cpu().numpy(), lse.cpu().numpy().astype(np.float64), q.numpy(), scale, k.decoded(), v.decoded(),
                  None if vis is None else vis.numpy(), (ok.decoded(), ov.decoded()) if own else None,
                  None if own_vis is None else own_vis.numpy(), B, M, H, G)


@pytest.mark.parametrize("T", [1, 2, 15, 31, 32, 33, 63, 64, 65, 100, 129, 500, 2047])
@pytest.mark.parametrize("D", [128, 96, 64])
def test_shared_prefix_lengths(T, D):
    _shared(1000 + T + D, 1, 5, 2, 4, T, D, 24 if D == 96 else 32)


@pytest.mark.parametrize("M,G", [(1, 1), (1, 16), (3, 4), (8, 2), (17, 1), (8, 4), (3, 11), (16, 4), (13, 5), (32, 4), (33, 4), (64, 4),
                                 (65, 4), (20, 16), (130, 4)])
@pytest.mark.parametrize("D", [128, 64])
def test_shared_query_rows(M, G, D):
    _shared(2000 + M * 16 + G + D, 1, M, 2, G, 333, D, 16, own=0)


@pytest.mark.parametrize("S,b_r", [(1, 1), (3, 8), (192, 4), (256, 6), (256, 8), (257, 6), (300, 4), (1024, 6), (2730, 8)])
@pytest.mark.parametrize("M", [3, 20])
def test_shared_codebooks(S, b_r, M):
    _shared(3000 + S + M, 1, M, 1, 4, 200, 128 if S % 2 else 64, S, b_r)


@pytest.mark.parametrize("B,M,H,G,T,D,own,limits,own_limits", [
    (2, 4, 3, 2, 300, 128, 40, None, None),
    (1, 6, 2, 4, 70, 96, 1, "ragged", "ragged"),
    (3, 5, 1, 8, 257, 64, 130, "some", "some"),
    (1, 2, 2, 1, 40, 128, 33, "none", "ragged"),
    (2, 3, 2, 2, 90, 64, 20, "none", "none"),
    (2, 40, 1, 4, 150, 128, 65, "ragged", "ragged"),
    (1, 1, 4, 4, 1000, 128, 200, None, "ragged"),
])
def test_shared_own_tokens_and_limits(B, M, H, G, T, D, own, limits, own_limits):
    _shared(4000 + T + own, B, M, H, G, T, D, 48, 4, own, limits, own_limits)


@pytest.mark.parametrize("M", [2, 30])
@pytest.mark.parametrize("Cmul,capacity,kgain,gain", [
    (0.3, None, 1.0, 1.0),     # nearly every chunk kept verbatim: windows longer than what is staged of them
    (1.2, None, 1.0, 1.0),
    (1.2, 37, 1.0, 1.0),       # the list too short: later payloads decode to zeros
    (3.0, 0, 1.0, 1.0),        # no list at all
    (3.0, None, 9000.0, 1e-3),  # scales at the end of the fp16 range: the reconstruction saturates
    (3.0, None, 1e-4, 3.0),    # tiny values
    (3.0, None, 1.0, 30.0),    # one-hot softmax
])
def test_shared_outliers_and_ranges(M, Cmul, capacity, kgain, gain):
    _shared(5000 + M, 1, M, 2, 4, 321, 128, 64, 6, own=30, Cmul=Cmul, capacity=capacity, kgain=kgain, gain=gain)


@pytest.mark.parametrize("M,own_T", [(2, 90), (2, 200), (140, 90), (40, 60)])
def test_shared_ignores_what_nobody_sees(M, own_T):
    """Payloads with NaN and infinities in tokens that no query head of a sequence sees, a sequence with NaN queries that sees
    nothing: the result is the one of clean caches, to the bit."""
    B, H, G, T, D, S = 1, 2, 4, 333, 128, 64
    N = B * M
    sk, sv = _secs(13, H, S)
    k, v = (Cache(1400 + i, B, H, T, D, s, Cmul=1.2) for i, s in enumerate((sk, sv)))
    ok, ov = (Cache(1410 + i, N, H, own_T, D, s, Cmul=1.2) for i, s in enumerate((sk, sv)))
    q = torch.randn(N, H * G, D, generator=_gen(1420)).to(torch.float16).to(DEV)
    most = 217  # of the prefix, by every query head of every sequence but the first, which sees nothing at all
    visible = torch.full((N, H * G), most, dtype=torch.int32, device=DEV)
    lengths = torch.randint(1, own_T - 3, (N, 1), generator=_gen(1430), dtype=torch.int32)
    lengths[0] = 0
    visible[0] = 0
    own_visible = lengths.expand(N, H * G).contiguous().to(DEV)
    ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(k.params, M, H * G, ok.params), dtype=torch.uint8, device=DEV)

    def run():
        out, lse = torch.full_like(q, float("nan")), torch.full((N, H * G), float("nan"), device=DEV)
        hq.hqmq_attend_shared(k.params, q, D ** -0.5, k.bufs, k.sec, v.bufs, v.sec, out, ws,
                              own=hq.OwnTokens(ok.params, ok.bufs, ov.bufs, own_visible), visible=visible, lse=lse)
        mass = torch.zeros(B, H, T, device=DEV)
        hq.hqmq_attend_mass(k.params, q, D ** -0.5, k.bufs, k.sec, lse, mass, visible=visible)
        torch.cuda.synchronize()
        return out.view(torch.int16).cpu(), lse.cpu(), mass.cpu()

    clean = run()
    assert torch.isfinite(clean[0].view(torch.float16)).all() and not clean[0][0].any()
    for c, limit in ((k, np.full(B, most)), (v, np.full(B, most)), (ok, lengths.numpy()[:, 0]), (ov, lengths.numpy()[:, 0])):
        off = c.bufs.row_off.cpu().numpy().view(np.uint32)
        pay = c.bufs.outliers.cpu().numpy().copy()
        flat = pay.reshape(-1, 4)
        for b in range(c.B):
            for h in range(H):
                r0 = (b * H + h) * c.T
                flat[off[r0 + limit[b]]:off[r0 + c.T]] = [np.nan, np.inf, -np.inf, 1.0]
        assert np.isnan(flat).any()
        c.bufs.outliers.copy_(torch.from_numpy(pay))
    q[0] = float("nan")
    for got, want in zip(run(), clean):
        assert torch.equal(got, want)


def test_shared_long_prefix():
    _shared(6000, 1, 9, 1, 4, 20011, 128, 256)
    _shared(6100, 1, 70, 1, 4, 9001, 64, 192, 4, own=17, limits="ragged")


@pytest.mark.parametrize("B,M,G,D,limits", [(100, 3, 2, 64, "ragged"), (140, 40, 2, 128, None), (130, 70, 2, 96, "some"), (140, 9, 3, 128, "ragged")])
def test_shared_one_share(B, M, G, D, limits):
    """As many heads as the chip holds: every workgroup has its rows' whole prefix and writes the result itself."""
    _shared(6400 + B + M, B, M, 8 if B == 100 else 2, G, 71, D, 16, 4, limits=limits)


def test_shared_most_parts():
    """One head: prefix and own tokens in 512 shares each, all of which the merge takes."""
    _shared(6300, 1, 1, 1, 2, 32768, 128, 32, own=32768)


def test_shared_long_own_tokens():
    """More own tokens than go with the prefix's launch."""
    _shared(6200, 1, 16, 1, 4, 50, 64, 48, 4, own=16500, own_limits="ragged")


def test_shared_with_one_sequence_is_attend():
    """n_share = 1 without own tokens is hqmq_attend_lse: the same value up to the rounding of both."""
    B, H, G, T, S = 2, 2, 4, 600, 64
    sk, sv = _secs(1, H, S)
    k, v = Cache(11, B, H, T, 128, sk), Cache(12, B, H, T, 128, sv)
    q = torch.randn(B, H * G, 128, generator=_gen(5)).to(torch.float16).to(DEV)
    o1, o2 = torch.empty_like(q), torch.empty_like(q)
    l1, l2 = (torch.empty(B, H * G, device=DEV) for _ in range(2))
    w1 = torch.empty(hq.hqmq_attend_workspace_bytes(k.params, H * G), dtype=torch.uint8, device=DEV)
    w2 = torch.empty(hq.hqmq_attend_shared_workspace_bytes(k.params, 1, H * G), dtype=torch.uint8, device=DEV)
    hq.hqmq_attend_lse(k.params, q, 0.09, k.bufs, k.sec, v.bufs, v.sec, o1, l1, w1)
    hq.hqmq_attend_shared(k.params, q, 0.09, k.bufs, k.sec, v.bufs, v.sec, o2, w2, lse=l2)
    torch.cuda.synchronize()
    assert (o1.float() - o2.float()).abs().max() <= 2 ** -9 * o1.float().abs().max()
    assert (l1 - l2).abs().max() < 1e-4


# ---- accumulated weight --------------------------------------------------------------------------------------------

def _mass(seed, B, M, H, G, T, D, S, b_r=6, decay=1.0, limits=None, in_place=False, Cmul=3.0, capacity=None, empty_rows=False,
          kgain=1.0, gain=1.0):
    sk, _ = _secs(seed, H, S)
    k = Cache(seed + 1, B, H, T, D, sk, b_r, Cmul, kgain, capacity)
    N = B * M
    q = (gain * torch.randn(N, H * G, D, generator=_gen(seed + 2))).to(torch.float16)
    vis = _limits(limits, N, H * G, T, seed + 3)
    lse = torch.randn(N, H * G, generator=_gen(seed + 4)) + math.log(T) + 1.0
    if empty_rows:
        lse[0, :] = float("-inf")
    mass = torch.rand(B, H, T, generator=_gen(seed + 5))
    m_dev = mass.to(DEV)
    if decay == 0.0:
        m_dev.fill_(float("nan"))  # is not read
    out = m_dev if in_place else torch.full_like(m_dev, float("nan"))
    scale = 1.0 / math.sqrt(D)
    hq.hqmq_attend_mass(k.params, q.to(DEV), scale, k.bufs, k.sec, lse.to(DEV), m_dev, decay=decay,
                        visible=None if vis is None else vis.to(DEV), out=None if in_place else out)
    torch.cuda.synchronize()
    K = k.decoded()
    s, delta, size = _scores(q.numpy(), K, scale, None if vis is None else vis.numpy(), B, M, H, G)
    l64 = _rows(lse.numpy().astype(np.float64), B, M, H, G)[..., None]
    w = np.where(np.isneginf(l64), 0.0, np.exp(s - np.where(np.isneginf(l64), 0.0, l64)))
    want = w.sum(2) + (decay * mass.numpy().astype(np.float64) if decay else 0.0)
    # an exponent is off by what roundings of K_hat move it, by the fp32 sum of D products (D 2^-24 of their magnitudes), and by
    # three fp32 roundings of score and lse in the log2 domain; exp2 is good to 2^-22; R fp32 additions and the last one
    R = M * G
    sf = np.where(np.isfinite(s), s, 0.0)
    e = 1.5 * delta + D * 2.0 ** -24 * size + 4 * 2.0 ** -24 * (np.abs(sf) + np.abs(np.where(np.isfinite(l64), l64, 0.0)))
    bound = (w * np.expm1(e)).sum(2) + (2.0 ** -22 + R * 2.0 ** -24) * w.sum(2) + 2.0 ** -23 * np.abs(want) + 1e-37
    got = out.cpu().numpy().astype(np.float64)
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), (np.argwhere(err > bound)[:5], err[err > bound][:5], bound[err > bound][:5])


@pytest.mark.parametrize("T", [1, 31, 32, 33, 64, 127, 513, 3000])
@pytest.mark.parametrize("D", [128, 96, 64])
def test_mass_lengths(T, D):
    _mass(7000 + T + D, 1, 1, 2, 4, T, D, 32)


@pytest.mark.parametrize("M,G", [(1, 1), (1, 16), (2, 4), (17, 1), (8, 4), (3, 11), (16, 4), (32, 4), (65, 4), (20, 16)])
def test_mass_query_rows(M, G):
    _mass(7500 + 16 * M + G, 2, M, 1, G, 211, 128 if M % 2 else 64, 16, 4)


@pytest.mark.parametrize("S,b_r", [(1, 1), (192, 4), (256, 6), (256, 8), (300, 4), (700, 6), (2730, 8)])
def test_mass_codebooks(S, b_r):
    _mass(7700 + S, 1, 3, 2, 4, 150, 128, S, b_r)


@pytest.mark.parametrize("kw", [
    dict(decay=0.0), dict(decay=0.0, limits="ragged"), dict(decay=0.75, in_place=True), dict(decay=-0.5),
    dict(limits="ragged"), dict(limits="some", empty_rows=True), dict(limits="none"), dict(empty_rows=True),
    dict(Cmul=0.3), dict(Cmul=1.2, capacity=37), dict(capacity=0), dict(kgain=9000.0, gain=1e-4), dict(kgain=1e-4),
])
@pytest.mark.parametrize("M", [1, 12])
def test_mass_states(kw, M):
    _mass(7900 + M, 2, M, 2, 4, 333, 128, 64, **kw)


@pytest.mark.parametrize("scale", [0.088, -0.125])
def test_mass_of_high_scores(scale):
    """Scores near 1000 and an lse beside them: a weight is off by the roundings of z = score - lse, not of the two.  With one
    element per query row the scores are exact, fma(score, scale, -lse) is off by 2^-24 |z|, its product with log2 e by 2^-24 |z|
    twice over (the constant, the product), and exp2 by 2^-22 of the weight."""
    H, T, D, d, c = 2, 700, 64, 5, 8192.0
    sk, _ = _secs(11, H, 64)
    k = Cache(71, 1, H, T, D, sk)
    K = k.decoded()
    scale = float(np.float32(scale))
    q = torch.zeros(1, H, D, dtype=torch.float16)
    q[..., d] = c
    s = scale * c * K.hat[0, :, :, d].astype(np.float64)
    lse = s.max(-1).astype(np.float32)
    assert (lse > 500).all()
    out = torch.empty(1, H, T, device=DEV)
    hq.hqmq_attend_mass(k.params, q.to(DEV), scale, k.bufs, k.sec, torch.from_numpy(lse)[None].to(DEV), None, decay=0.0, out=out)
    z = s - lse.astype(np.float64)[:, None]
    want, sure = np.exp(z), K.slack[0, :, :, d] == 0
    err, bound = np.abs(out.cpu().numpy()[0] - want), (3 * 2.0 ** -24 * np.abs(z) + 2.0 ** -22) * want * 1.01 + 2.0 ** -126
    assert sure.any() and (err <= bound)[sure].all(), (err[sure].max(), np.argwhere(sure & (err > bound))[:5])


def test_mass_sums_to_the_rows():
    """With the lse that the attention returned, every query row's weights sum to one."""
    B, M, H, G, T, S = 1, 6, 2, 4, 900, 64
    sk, sv = _secs(3, H, S)
    k, v = Cache(31, B, H, T, 128, sk), Cache(32, B, H, T, 128, sv)
    q = (2 * torch.randn(B * M, H * G, 128, generator=_gen(33))).to(torch.float16).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(B * M, H * G, device=DEV)
    ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(k.params, M, H * G), dtype=torch.uint8, device=DEV)
    hq.hqmq_attend_shared(k.params, q, 0.088, k.bufs, k.sec, v.bufs, v.sec, out, ws, lse=lse)
    mass = torch.empty(B, H, T, device=DEV)
    hq.hqmq_attend_mass(k.params, q, 0.088, k.bufs, k.sec, lse, None, decay=0.0, out=mass)
    assert (mass.double().sum(-1) - M * G).abs().max().item() < 1e-3


# ---- the choice of the tokens ----------------------------------------------------------------------------------------

def _select_reference(mass, lengths, n_sink, n_recent, n_keep):
    B, H, T = mass.shape
    keep = np.full((B, H, n_keep), -1, np.int32)
    n_kept = np.zeros((B, H), np.int32)
    for b in range(B):
        L = T if lengths is None else min(max(int(lengths[b]), 0), T)
        for h in range(H):
            if L <= n_keep:
                kept = np.arange(L)
            else:
                m = np.where(np.isnan(mass[b, h]), -np.inf, mass[b, h]).astype(np.float64)
                mid = np.arange(n_sink, L - n_recent)
                nan_last = np.isnan(mass[b, h, mid])
                order = mid[np.lexsort((mid, -m[mid], nan_last))]
                kept = np.sort(np.concatenate([np.arange(n_sink), order[: n_keep - n_sink - n_recent], np.arange(L - n_recent, L)]))
            keep[b, h, : len(kept)] = kept
            n_kept[b, h] = len(kept)
    return keep, n_kept


def _select(mass, n_keep, n_sink, n_recent, lengths=None, with_mass=True):
    B, H, T = mass.shape
    m = torch.from_numpy(mass).to(DEV)
    keep = torch.full((B, H, n_keep), -7, dtype=torch.int32, device=DEV)
    n_kept = torch.full((B, H), -7, dtype=torch.int32, device=DEV)
    km = torch.full((B, H, n_keep), float("nan"), device=DEV) if with_mass else None
    ws = torch.empty(max(1, hq.hqmq_evict_select_workspace_bytes(B, H, T, n_keep)), dtype=torch.uint8, device=DEV)
    ws.fill_(0xCD)
    hq.hqmq_evict_select(m, n_sink, n_recent, keep, n_kept, ws, None if lengths is None else torch.tensor(lengths, dtype=torch.int32).to(DEV), km)
    torch.cuda.synchronize()
    want, n = _select_reference(mass, lengths, n_sink, n_recent, n_keep)
    assert np.array_equal(n_kept.cpu().numpy(), n)
    assert np.array_equal(keep.cpu().numpy(), want)
    if with_mass:
        wm = np.where(want >= 0, np.take_along_axis(mass, np.maximum(want, 0), 2), np.float32(0))
        assert np.array_equal(km.cpu().numpy().view(np.uint32), wm.view(np.uint32))


def _values(kind, shape, seed):
    r = np.random.RandomState(seed)
    x = np.exp(2 * r.randn(*shape)).astype(np.float32)
    if kind == "ties":
        x = r.randint(0, 4, shape).astype(np.float32)
    elif kind == "equal":
        x[:] = 0.25
    elif kind == "zeros":
        x[r.rand(*shape) < 0.7] = 0.0
        x[r.rand(*shape) < 0.3] = -0.0
    elif kind == "odd":
        x = r.randn(*shape).astype(np.float32)
        for v in (np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38):
            x[r.rand(*shape) < 0.08] = v
    elif kind == "close":  # neighbours in the last bits
        x = (np.float32(1.5).view(np.uint32) + r.randint(0, 5, shape).astype(np.uint32)).view(np.float32)
    elif kind == "rising":
        x = np.broadcast_to(np.arange(shape[-1], dtype=np.float32), shape).copy()
    elif kind == "falling":
        x = np.broadcast_to(-np.arange(shape[-1], dtype=np.float32), shape).copy()
    return x


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "zeros", "odd", "close", "rising", "falling"])
@pytest.mark.parametrize("B,H,T,n_keep,n_sink,n_recent", [
    (1, 1, 1, 1, 0, 0), (1, 2, 2, 1, 0, 0), (1, 3, 65, 64, 4, 10), (2, 2, 1000, 333, 4, 32), (1, 2, 1025, 1, 1, 0),
    (1, 2, 4097, 2048, 0, 0), (1, 1, 5000, 4999, 3, 5), (1, 1, 9001, 100, 60, 40), (3, 1, 12345, 1234, 4, 128),
])
def test_select(kind, B, H, T, n_keep, n_sink, n_recent):
    _select(_values(kind, (B, H, T), T + n_keep), n_keep, n_sink, n_recent)


@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
@pytest.mark.parametrize("T,n_keep", [(32768, 4096), (70001, 7000), (131072, 1)])
def test_select_long(kind, T, n_keep):
    _select(_values(kind, (1, 2, T), T), n_keep, min(4, n_keep - 1), 0)


@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_select_ragged(kind):
    lengths = [0, 1, 63, 64, 65, 700, 1999, 2000, 2001, -4, 300]
    _select(_values(kind, (len(lengths), 2, 2000), 3), 64, 3, 20, lengths)
    _select(_values(kind, (len(lengths), 2, 2000), 4), 2000, 0, 0, lengths, with_mass=False)
    _select(_values(kind, (3, 2, 20000), 4), 3000, 4, 100, [20000, 2999, 9000])


@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "zeros", "equal"])
@pytest.mark.parametrize("n_keep,n_sink,n_recent", [(3000, 4, 100), (36000, 0, 1), (1, 0, 0)])
def test_select_ragged_long(kind, n_keep, n_sink, n_recent):
    """Heads that several workgroups share: lengths that end in the first of them, between two, and that keep everything."""
    lengths = [40000, 33000, 8192, 8193, 100, 0, 3000]
    _select(_values(kind, (len(lengths), 2, 40000), 5), n_keep, n_sink, n_recent, lengths)


@pytest.mark.parametrize("kind", ["spread", "ties", "equal"])
def test_select_many_tokens(kind):
    """More tokens than 64 workgroups take in one piece each: three pieces, the last ones short or empty."""
    _select(_values(kind, (3, 1, 1100003), 6), 5000, 4, 64, [1100003, 600000, 4999])


def test_select_many_heads():
    _select(_values("spread", (40, 32, 257), 9), 64, 4, 16)


# ---- compaction ------------------------------------------------------------------------------------------------------

def _empty_like(params, n_keep, capacity):
    p = hq.compacted_params(params, n_keep)
    e = hq.alloc_encoded(p, DEV, capacity)
    for t in (e.codes, e.flags, e.row_off, e.n_outliers, e.status):
        t.fill_(-9)
    e.sigma.fill_(7.0)
    e.outliers.fill_(7.0)
    return e


def _compact_reference(bufs, p, keep, capacity):
    """The new tensor's parts, numpy; list entries that nothing writes stay 7.0."""
    u32 = lambda t: t.cpu().numpy().view(np.uint32)  # noqa: E731
    codes, flags, off = u32(bufs.codes), u32(bufs.flags), u32(bufs.row_off)
    sigma = bufs.sigma.cpu().numpy().view(np.uint16)
    outl = bufs.outliers.cpu().numpy().view(np.uint16).reshape(-1, 4)
    B, H, n = keep.shape
    rows = (np.arange(B * H).reshape(B, H, 1) * p.T + keep).reshape(-1)
    there = ((keep >= 0) & (keep < p.T)).reshape(-1)
    rows = np.where(there, rows, 0)
    f = np.where(there, flags[rows], 0).astype(np.uint32)
    cnt = np.array([bin(int(x)).count("1") for x in f])
    new_off = np.concatenate([[0], np.cumsum(cnt)]).astype(np.uint32)
    new_outl = np.full((capacity, 4), np.float16(7.0)).view(np.uint16)
    for i, (r, c, o) in enumerate(zip(rows, cnt, new_off[:-1])):
        for j in range(c):
            if o + j < capacity:
                src = int(off[r]) + j
                new_outl[o + j] = outl[src] if src < len(outl) else 0
    heads = cnt.reshape(B, H, n).sum((0, 2))
    status = int(bufs.status.cpu().numpy().view(np.uint32)[0]) | (1 if new_off[-1] > capacity else 0)
    return {"codes": np.where(there[:, None], codes[rows], 0).astype(np.uint32), "sigma": np.where(there, sigma[rows], 0).astype(np.uint16),
            "flags": f, "row_off": new_off, "outliers": new_outl, "n_outliers": np.append(heads, heads.sum()).astype(np.uint32),
            "status": np.array([status], np.uint32)}


def _assert_compacted(out, want):
    for name, w in want.items():
        t = getattr(out, name).cpu().numpy()
        got = t.view(np.uint16 if t.dtype == np.float16 else np.uint32)
        assert np.array_equal(got.reshape(w.shape), w), name


def _compact(seed, n, B, H, T, D, n_keep, S=24, b_r=6, Cmul=2.0, in_cap=None, out_cap=None, order="sorted", short=False):
    caches = [Cache(seed + i, B, H, T, D, _secs(seed + i, H, S)[0], b_r, Cmul, capacity=in_cap) for i in range(n)]
    r = np.random.RandomState(seed)
    keeps = []
    for i in range(n):
        if order == "any":      # repeats, no order, indices outside
            keep = r.randint(-3, T + 3, (B, H, n_keep))
            keep[0, 0, 0] = np.iinfo(np.int32).min
            keep[-1, -1, -1] = np.iinfo(np.int32).max
        else:
            keep = np.stack([np.sort(r.permutation(T)[:n_keep]) for _ in range(B * H)]).reshape(B, H, n_keep)
        if short:
            keep = np.where(np.arange(n_keep) < r.randint(0, n_keep + 1, (B, H, 1)), keep, -1)
        keeps.append(keep.astype(np.int32))
    p = caches[0].params
    cap = B * H * n_keep * ((D + 3) // 4) + 3 if out_cap is None else out_cap
    outs = [_empty_like(p, n_keep, cap) for _ in range(n)]
    ws = torch.empty(hq.hqmq_evict_compact_workspace_bytes(p, n_keep, n), dtype=torch.uint8, device=DEV)
    ws.fill_(0xCD)
    hq.hqmq_evict_compact(hq.CompactBatch(p, [c.bufs for c in caches], [torch.from_numpy(k).to(DEV) for k in keeps], outs, ws))
    torch.cuda.synchronize()
    for c, k, o in zip(caches, keeps, outs):
        _assert_compacted(o, _compact_reference(c.bufs, p, k, cap))
    return caches, keeps, outs


@pytest.mark.parametrize("B,H,T,D,n_keep", [
    (1, 1, 1, 128, 1), (1, 2, 300, 128, 77), (2, 3, 513, 96, 256), (1, 2, 700, 64, 257), (3, 5, 337, 100, 101), (1, 1, 900, 45, 600),
    (2, 2, 100, 4, 99), (1, 2, 65, 1, 33), (1, 8, 3000, 128, 1025), (70, 3, 40, 64, 9),
])
def test_compact(B, H, T, D, n_keep):
    _compact(8000 + T + D, 2, B, H, T, D, n_keep, S=24 if D % 2 else 256, b_r=3 if D == 100 else 6)


@pytest.mark.parametrize("kw", [
    dict(order="any"), dict(short=True), dict(order="any", n_keep=500), dict(in_cap=11), dict(in_cap=0), dict(out_cap=0), dict(out_cap=23),
    dict(in_cap=50, out_cap=60, order="any"), dict(Cmul=0.2), dict(Cmul=100.0),
])
def test_compact_states(kw):
    _compact(8500, 1, **{**dict(B=2, H=3, T=290, D=128, n_keep=120), **kw})


def test_compact_many_heads():
    """More counts than are summed directly: 4200 and 8400 blocks of 256 rows."""
    _compact(8600, 2, 600, 7, 4, 64, 3, order="any")
    _compact(8650, 1, 300, 14, 4, 64, 257, order="any")


@pytest.mark.parametrize("n", [24, 25, 60])
def test_compact_many_tensors(n):
    _compact(8700, n, 1, 2, 40, 64, 11)


def test_compacted_rows_decode_as_before():
    caches, keeps, outs = _compact(8800, 1, 2, 2, 400, 128, 150)
    c, keep, o = caches[0], keeps[0], outs[0]
    full, part = torch.empty(2, 2, 400, 128, dtype=torch.float16, device=DEV), torch.empty(2, 2, 150, 128, dtype=torch.float16, device=DEV)
    hq.hqmq_decode(c.params, c.bufs, c.sec, full)
    hq.hqmq_decode(hq.compacted_params(c.params, 150), o, c.sec, part)
    idx = torch.from_numpy(keep).long().to(DEV).unsqueeze(-1).expand(-1, -1, -1, 128)
    assert torch.equal(full.gather(2, idx).view(torch.int16), part.view(torch.int16))


# ---- together --------------------------------------------------------------------------------------------------------

class Serving:
    """A generation step over a shared prefix and own tokens, the weights' sums of both, and the own tokens trimmed to a
    budget: the calls in the order in which a server makes them, on buffers made once."""

    def __init__(self, seed=9000, B=1, M=3, H=2, G=4, T=700, own=300, D=128, S=64, budget=100):
        self.B, self.M, self.H, self.G, self.D, self.scale = B, M, H, G, D, D ** -0.5
        N = B * M
        sk, sv = _secs(seed, H, S)
        self.k, self.v = Cache(seed + 1, B, H, T, D, sk), Cache(seed + 2, B, H, T, D, sv)
        self.ok, self.ov = Cache(seed + 3, N, H, own, D, sk), Cache(seed + 4, N, H, own, D, sv)
        self.q = (1.5 * torch.randn(N, H * G, D, generator=_gen(seed + 5))).to(torch.float16).to(DEV)
        self.lengths = torch.tensor([own, own - 57, 40][:N] + [own] * max(0, N - 3), dtype=torch.int32).to(DEV)
        self.visible = self.lengths.view(N, 1).expand(N, H * G).contiguous()
        f32 = dict(dtype=torch.float32, device=DEV)
        self.mass, self.own_mass = torch.zeros(B, H, T, **f32), torch.zeros(N, H, own, **f32)
        self.out, self.lse = torch.empty_like(self.q), torch.empty(N, H * G, **f32)
        self.tokens = hq.OwnTokens(self.ok.params, self.ok.bufs, self.ov.bufs, self.visible)
        self.ws = torch.empty(hq.hqmq_attend_shared_workspace_bytes(self.k.params, M, H * G, self.ok.params), dtype=torch.uint8, device=DEV)
        self.keep = torch.empty(N, H, budget, dtype=torch.int32, device=DEV)
        self.n_kept = torch.empty(N, H, dtype=torch.int32, device=DEV)
        self.kept_mass = torch.empty(N, H, budget, **f32)
        self.sws = torch.empty(max(1, hq.hqmq_evict_select_workspace_bytes(N, H, own, budget)), dtype=torch.uint8, device=DEV)
        p = self.ok.params
        self.small = [hq.alloc_encoded(hq.compacted_params(p, budget), DEV, N * H * budget * 8) for _ in range(2)]
        self.cws = torch.empty(hq.hqmq_evict_compact_workspace_bytes(p, budget, 2), dtype=torch.uint8, device=DEV)
        self.batch = hq.CompactBatch(p, [self.ok.bufs, self.ov.bufs], [self.keep] * 2, self.small, self.cws)
        self.small_visible = torch.empty_like(self.visible)
        self.small_tokens = hq.OwnTokens(hq.compacted_params(p, budget), self.small[0], self.small[1], self.small_visible)
        self.out2, self.lse2 = torch.empty_like(self.q), torch.empty_like(self.lse)

    def step(self):
        a = (self.k.params, self.q, self.scale, self.k.bufs, self.k.sec, self.v.bufs, self.v.sec)
        hq.hqmq_attend_shared(*a, self.out, self.ws, own=self.tokens, lse=self.lse)
        hq.hqmq_attend_mass(self.k.params, self.q, self.scale, self.k.bufs, self.k.sec, self.lse, self.mass, decay=0.5)
        hq.hqmq_attend_mass(self.ok.params, self.q, self.scale, self.ok.bufs, self.ok.sec, self.lse, self.own_mass, visible=self.visible)
        hq.hqmq_evict_select(self.own_mass, 2, 16, self.keep, self.n_kept, self.sws, self.lengths, self.kept_mass)
        hq.hqmq_evict_compact(self.batch)
        self.small_visible.copy_(self.n_kept.repeat_interleave(self.G, 1))
        hq.hqmq_attend_shared(*a, self.out2, self.ws, own=self.small_tokens, lse=self.lse2)

    def results(self):
        total = int(self.small[0].n_outliers[-1]), int(self.small[1].n_outliers[-1])
        parts = [t for e in self.small for t in (e.codes, e.sigma, e.flags, e.row_off, e.n_outliers, e.status)]
        return [t.clone().view(torch.int16 if t.dtype == torch.float16 else torch.int32)
                for t in [self.out, self.lse, self.mass, self.own_mass, self.keep, self.n_kept, self.kept_mass, self.out2, self.lse2, *parts,
                          *(e.outliers[:n] for e, n in zip(self.small, total))]]

    def scrub(self):
        for t in (self.out, self.lse, self.out2, self.lse2, self.kept_mass):
            t.fill_(float("nan"))
        for t in (self.keep, self.n_kept, *(x for e in self.small for x in (e.codes, e.flags, e.row_off, e.n_outliers, e.status))):
            t.fill_(-5)
        for t in (self.ws, self.sws, self.cws):
            t.fill_(0x77)
        self.mass.zero_()
        self.own_mass.zero_()


def test_serving_step():
    """The whole sequence against the references: outputs over the whole and the trimmed caches, weights, choice, rows."""
    s = Serving()
    s.step()
    torch.cuda.synchronize()
    q, lens = s.q.cpu().numpy(), s.visible.cpu().numpy()
    K, V, OK, OV = s.k.decoded(), s.v.decoded(), s.ok.decoded(), s.ov.decoded()
    dims = (s.B, s.M, s.H, s.G)
    _check_shared(s.out.cpu().numpy(), s.lse.cpu().numpy().astype(np.float64), q, s.scale, K, V, None, (OK, OV), lens, *dims)
    own_mass = s.own_mass.cpu().numpy()
    keep, n_kept = _select_reference(own_mass, s.lengths.cpu().numpy(), 2, 16, s.keep.shape[2])
    assert np.array_equal(s.keep.cpu().numpy(), keep) and np.array_equal(s.n_kept.cpu().numpy(), n_kept)
    for c, o in ((s.ok, s.small[0]), (s.ov, s.small[1])):
        want = _compact_reference(c.bufs, c.params, keep, o.outlier_capacity)
        want["outliers"] = want["outliers"][: int(want["row_off"][-1])]
        got = hq.EncodedBuffers(o.codes, o.sigma, o.flags, o.row_off, o.outliers[: len(want["outliers"])], o.n_outliers, o.status)
        _assert_compacted(got, want)
    sk, sv = s.ok.sec_np, s.ov.sec_np
    p = hq.compacted_params(s.ok.params, keep.shape[2])
    trimmed = decoded_of(s.small[0], p, sk), decoded_of(s.small[1], p, sv)
    _check_shared(s.out2.cpu().numpy(), s.lse2.cpu().numpy().astype(np.float64), q, s.scale, K, V, None, trimmed,
                  np.repeat(n_kept, s.G, 1), *dims)
    # every query row's weights over prefix and own tokens sum to one
    total = s.mass.cpu().numpy().sum(-1).sum() + own_mass.sum()
    assert abs(total - s.B * s.M * s.H * s.G) < 1e-2


@pytest.mark.parametrize("kw", [dict(M=20, T=500, own=130, D=64, S=24), dict(M=3, T=500, own=33000, D=64, S=24)])
def test_serving_graph_replays(kw):
    """A short step, and one whose own tokens are chosen from by several workgroups per head."""
    s = Serving(9500, **kw)
    hq.hqmq_init()
    s.scrub()
    s.step()
    torch.cuda.synchronize()
    want = s.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.scrub()
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.step()
    for rep in range(3):
        s.scrub()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(s.results(), want):
            assert torch.equal(a, b), rep
        s.scrub()
        s.step()  # the program's own eager work between the replays
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Two calls in flight on streams of their own, with their own workspaces."""
    a, b = Serving(9600), Serving(9700, M=18, T=900, D=96, S=24)
    for s in (a, b):
        s.scrub()
        s.step()
    torch.cuda.synchronize()
    want = a.results(), b.results()
    for s in (a, b):
        s.scrub()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, st in zip((a, b), streams):
        with torch.cuda.stream(st):
            s.step()
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        for x, y in zip(s.results(), w):
            assert torch.equal(x, y)
