"""Edges of the calls that serve a batch from packed caches, beside test_gpu_serve.py and with its helpers: keys that are not
finite, limits far outside, weights' bits, and the forms of each kernel."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2605_27646_amd as hq
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
