"""Host-side checks of include/hqmq_serve.h that need no GPU: the library exports what the header declares and refuses bad
arguments before anything is enqueued (pointers here are addresses that are never read)."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2605_27646_amd as hq
from paper_2605_27646_amd import binding, serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an aligned address
INVALID, UNSUPPORTED, SMALL = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hq.library_path()):
        from paper_2605_27646_amd import build
        build.build()
    return serving._load()


def _params(**kw):
    d = dict(B=2, H=4, T=1000, D=128, stride_b=4 * 1000 * 128, stride_h=1000 * 128, stride_t=128, S=64, b_r=6, C=3.0, flags=0)
    d.update(kw)
    return hq.HqmqParams(**d)


def _enc(base=P, **kw):
    names = ("codes", "sigma", "flags", "row_off", "outliers", "n_outliers", "status")
    at = {n: base + 4096 * i for i, n in enumerate(names)}
    at.update(kw)
    return binding._Encoded(*[at[n] for n in names])


def test_header_and_library_agree(lib):
    header = open(os.path.join(ROOT, "include", "hqmq_serve.h")).read()
    declared = set(re.findall(r"^(?:int32_t|uint64_t)\s+(hqmq_\w+)\s*\(", header, re.M))
    assert declared == {"hqmq_attend_shared", "hqmq_attend_shared_workspace_bytes", "hqmq_attend_mass", "hqmq_evict_select",
                        "hqmq_evict_select_workspace_bytes", "hqmq_evict_compact", "hqmq_evict_compact_workspace_bytes"}
    for name in declared:
        assert hasattr(lib, name) and hasattr(hq, name), name
    assert C.sizeof(serving._Own) == 48
    assert int(re.search(r"#define HQMQ_MAX_SHARE (\d+)", header).group(1)) == hq.HQMQ_MAX_SHARE


def _shared(lib, params=None, n_share=3, heads=8, q=P, scale=0.1, enc_k=None, cap_k=5, sec=P, enc_v=None, vis=0, own=None, out=P, lse=0,
            ws=P, ws_bytes=1 << 40):
    params = _params() if params is None else params
    enc_k, enc_v = enc_k or _enc(), enc_v or _enc()
    return lib.hqmq_attend_shared(C.byref(params), n_share, heads, q, scale, C.byref(enc_k), cap_k, sec, C.byref(enc_v), 5, sec, vis or None,
                                  None if own is None else C.byref(own), out, lse or None, ws, ws_bytes, None)


def _own(params, enc_k=None, enc_v=None, vis=0):
    ek, ev = enc_k or _enc(), enc_v or _enc()
    o = serving._Own(C.pointer(params), C.pointer(ek), C.pointer(ev), 5, 5, vis or None)
    o.refs = (params, ek, ev)
    return o


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(n_share=0)), (INVALID, dict(n_share=-1)), (INVALID, dict(n_share=1025)), (INVALID, dict(heads=6)), (INVALID, dict(heads=0)),
    (UNSUPPORTED, dict(heads=4 * 17)), (UNSUPPORTED, dict(params=_params(D=100))), (UNSUPPORTED, dict(params=_params(S=2731))),
    (UNSUPPORTED, dict(params=_params(b_r=9))), (INVALID, dict(params=_params(T=0))),
    (UNSUPPORTED, dict(params=_params(B=64), n_share=1024, heads=4)),
    (INVALID, dict(q=None)), (INVALID, dict(q=P + 8)), (INVALID, dict(out=None)), (INVALID, dict(out=P + 2)), (INVALID, dict(sec=None)),
    (INVALID, dict(sec=P + 4)), (INVALID, dict(ws=None)), (INVALID, dict(ws=P + 128)), (INVALID, dict(vis=P + 2)), (INVALID, dict(lse=P + 1)),
    (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (SMALL, dict(ws_bytes=1000)),
    (INVALID, dict(enc_k=_enc(codes=0))), (INVALID, dict(enc_v=_enc(row_off=P + 2))), (INVALID, dict(enc_k=_enc(outliers=0))),
    (INVALID, dict(own=_own(_params(B=5)))), (INVALID, dict(own=_own(_params(B=6, H=8)))), (INVALID, dict(own=_own(_params(B=6, S=32)))),
    (INVALID, dict(own=_own(_params(B=6, b_r=4)))), (INVALID, dict(own=_own(_params(B=6, D=64)))), (INVALID, dict(own=_own(_params(B=6, T=0)))),
    (INVALID, dict(own=_own(_params(B=6), enc_k=_enc(flags=0)))), (INVALID, dict(own=_own(_params(B=6), vis=P + 1))),
    (INVALID, dict(own=serving._Own())),
])
def test_shared_refuses(lib, want, kw):
    assert _shared(lib, **kw) == want


def test_shared_workspace(lib):
    p = _params()
    assert hq.hqmq_attend_shared_workspace_bytes(p, 0, 8) == 0 and hq.hqmq_attend_shared_workspace_bytes(p, 3, 7) == 0
    assert hq.hqmq_attend_shared_workspace_bytes(p, 3, 8, _params(B=5)) == 0
    alone, both = (hq.hqmq_attend_shared_workspace_bytes(p, 3, 8, o) for o in (None, _params(B=6, T=100)))
    assert 0 < alone < both and alone % 256 == both % 256 == 0
    assert _shared(lib, ws_bytes=alone - 1) == SMALL
    assert _shared(lib, own=_own(_params(B=6, T=100)), ws_bytes=both - 1) == SMALL


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(n_share=0)), (INVALID, dict(n_share=2000)), (INVALID, dict(heads=9)), (UNSUPPORTED, dict(params=_params(D=92))),
    (INVALID, dict(q=None)), (INVALID, dict(q=P + 4)), (INVALID, dict(sec=None)), (INVALID, dict(lse=None)), (INVALID, dict(lse=P + 2)),
    (INVALID, dict(vis=P + 2)), (INVALID, dict(mass=None)), (INVALID, dict(mass=P + 2)), (INVALID, dict(out=None)), (INVALID, dict(out=P + 2)),
    (INVALID, dict(decay=float("nan"))), (INVALID, dict(decay=float("inf"))), (INVALID, dict(scale=float("nan"))), (INVALID, dict(enc=_enc(sigma=0))),
])
def test_mass_refuses(lib, want, kw):
    a = dict(params=_params(), n_share=3, heads=8, q=P, scale=0.1, enc=_enc(), sec=P, lse=P, vis=None, mass=P, decay=1.0, out=P)
    a.update(kw)
    assert lib.hqmq_attend_mass(C.byref(a["params"]), a["n_share"], a["heads"], a["q"], a["scale"], C.byref(a["enc"]), 5, a["sec"], a["lse"],
                                a["vis"], a["mass"], a["decay"], a["out"], None) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(B=0)), (INVALID, dict(H=-1)), (INVALID, dict(T=0)), (INVALID, dict(n_keep=0)), (INVALID, dict(n_keep=1001)),
    (INVALID, dict(n_sink=-1)), (INVALID, dict(n_recent=-1)), (INVALID, dict(n_sink=101)), (INVALID, dict(n_sink=50, n_recent=51)),
    (INVALID, dict(n_sink=2 ** 31 - 1, n_recent=2 ** 31 - 1)), (UNSUPPORTED, dict(B=70000, T=100)), (UNSUPPORTED, dict(B=4, H=4, T=1 << 28)),
    (INVALID, dict(mass=None)), (INVALID, dict(mass=P + 2)), (INVALID, dict(keep=None)), (INVALID, dict(keep=P + 1)), (INVALID, dict(kept=None)),
    (INVALID, dict(kept=P + 1)), (INVALID, dict(length=P + 2)), (INVALID, dict(km=P + 2)), (INVALID, dict(ws=P + 8)),
])
def test_select_refuses(lib, want, kw):
    a = dict(B=2, H=4, T=1000, mass=P, length=None, n_sink=2, n_recent=3, n_keep=100, keep=P, kept=P, km=None, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    assert lib.hqmq_evict_select(a["B"], a["H"], a["T"], a["mass"], a["length"], a["n_sink"], a["n_recent"], a["n_keep"], a["keep"], a["kept"],
                                 a["km"], a["ws"], a["ws_bytes"], None) == want


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(n=0)), (INVALID, dict(n=-2)), (INVALID, dict(n_keep=0)), (UNSUPPORTED, dict(n_keep=1 << 28)), (UNSUPPORTED, dict(params=_params(D=129, stride_t=130))),
    (INVALID, dict(ws=None)), (INVALID, dict(ws=P + 64)), (SMALL, dict(ws_bytes=16)), (INVALID, dict(keep=None)), (INVALID, dict(keep=P + 2)),
    (INVALID, dict(enc=_enc(status=0))), (INVALID, dict(enc=_enc(codes=0))), (INVALID, dict(out=_enc(2 * P, n_outliers=0))),
    (INVALID, dict(out=_enc(2 * P, status=0))), (INVALID, dict(out=_enc(P))), (INVALID, dict(out=_enc(2 * P, codes=P))),
    (INVALID, dict(out=_enc(2 * P, outliers=0))),
])
def test_compact_refuses(lib, want, kw):
    a = dict(params=_params(), n_keep=100, n=1, enc=_enc(), keep=P, out=_enc(2 * P), ws=P, ws_bytes=1 << 40)
    a.update(kw)
    one, keep = (C.c_uint64 * 1)(5), (C.c_void_p * 1)(a["keep"])
    assert lib.hqmq_evict_compact(C.byref(a["params"]), a["n_keep"], a["n"], C.byref(a["enc"]), one, keep, C.byref(a["out"]), one, a["ws"],
                                  a["ws_bytes"], None) == want


def test_compact_refuses_one_buffer_twice(lib):
    """Two of the new tensors in one place, or one where another is still read."""
    params, caps, keep = _params(), (C.c_uint64 * 2)(5, 5), (C.c_void_p * 2)(P, P)
    enc = (binding._Encoded * 2)(_enc(P), _enc(2 * P))
    for outs in ((_enc(3 * P), _enc(3 * P)), (_enc(2 * P), _enc(4 * P)), (_enc(3 * P), _enc(4 * P, sigma=P + 4096))):
        out = (binding._Encoded * 2)(*outs)
        assert lib.hqmq_evict_compact(C.byref(params), 10, 2, enc, caps, keep, out, caps, P, 1 << 40, None) == INVALID


def test_workspaces_of_invalid_arguments_are_zero():
    assert hq.hqmq_evict_select_workspace_bytes(0, 1, 1, 1) == 0 and hq.hqmq_evict_select_workspace_bytes(1, 1, 5, 6) == 0
    assert hq.hqmq_evict_compact_workspace_bytes(_params(), 0, 1) == 0 and hq.hqmq_evict_compact_workspace_bytes(_params(), 10, 0) == 0
    assert hq.hqmq_evict_compact_workspace_bytes(_params(), 10, 1) > 0


def test_compacted_params():
    p = hq.compacted_params(_params(flags=1), 37)
    assert (p.B, p.H, p.T, p.D, p.stride_t, p.stride_h, p.stride_b, p.S, p.b_r, p.flags) == (2, 4, 37, 128, 128, 37 * 128, 4 * 37 * 128, 64, 6, 1)


def test_binding_refuses_shapes():
    """Shapes and types are checked before the library is called."""
    p = _params()
    q = torch.zeros(6, 8, 128, dtype=torch.float16)
    for bad in (q.float(), q[:5], q[:, :, :64].contiguous(), q[0], q[:, ::2], q[:0]):
        with pytest.raises(ValueError):
            serving._share_of(p, bad)
    assert serving._share_of(p, q) == 3
    for bad in (torch.zeros(2, 3), torch.zeros(2, 4, dtype=torch.float64), torch.zeros(4, 4)[::2]):
        with pytest.raises(ValueError):
            serving._rows_of("x", bad, torch.float32, (2, 4))
    m = torch.zeros(2, 4, 1000)
    with pytest.raises(ValueError):
        hq.hqmq_attend_mass(p, q, 0.1, None, None, None, None)
    with pytest.raises(ValueError):
        hq.hqmq_attend_mass(p, q, 0.1, None, None, torch.zeros(6, 8), m[:, :, :-1])
    with pytest.raises(ValueError):
        hq.hqmq_evict_select(m[0], 0, 0, torch.zeros(2, 4, 5, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        hq.hqmq_evict_select(m, 0, 0, torch.zeros(2, 3, 5, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        hq.CompactBatch(p, [], [], [], torch.zeros(1))


def test_select_refuses_too_many_tokens(lib):
    assert lib.hqmq_evict_select(1, 1, (1 << 30) + 1, P, None, 0, 0, 1, P, P, None, P, 1 << 60, None) == UNSUPPORTED
    assert hq.hqmq_evict_select_workspace_bytes(1, 1, (1 << 30) + 1, 1) == 0 and hq.hqmq_evict_select_workspace_bytes(1, 1, 1 << 30, 1) > 0


def test_own_tokens_refuse_short_buffers():
    """Buffers of fewer rows than params says are refused where the sequences' tokens are put together."""
    p, fewer = _params(), _params(T=900, stride_b=4 * 900 * 128, stride_h=900 * 128)
    full, short = hq.alloc_encoded(p, "cpu", 10), hq.alloc_encoded(fewer, "cpu", 10)
    assert hq.OwnTokens(p, full, full).struct.cap_k == 10
    for k, v in ((full, short), (short, full)):
        with pytest.raises(ValueError):
            hq.OwnTokens(p, k, v)


LIMITS = """
#include <climits>
#include "hqmq_limits.h"
using namespace hqmq;
constexpr int smaller(int a, int b) { return a < b ? a : b; }
// rows of the tile that wave `wave` of a split begins with, of tokens of which the heads' largest limit is `most`
constexpr int first_rows(int T, int begin, int wave, int most) { return tile_rows(smaller(T, seen_tokens(most)), begin + 16 * wave, 16); }
static_assert(seen_tokens(INT_MIN) == 0 && seen_tokens(-1) == 0 && seen_tokens(0) == 0 && seen_tokens(7) == 7 && seen_tokens(INT_MAX) == INT_MAX, "");
static_assert(first_rows(1, 0, 3, INT_MIN) <= 0 && first_rows(1 << 27, (1 << 27) - 64, 7, INT_MIN) <= 0 && first_rows(1, 0, 0, INT_MIN) <= 0, "");
static_assert(first_rows(100, 64, 0, INT_MAX) == 16 && first_rows(100, 64, 2, 1000) == 4 && first_rows(100, 64, 3, 1000) <= 0, "");
static_assert(first_rows(100, 64, 0, 70) == 6 && first_rows(100, 64, 1, 70) <= 0, "");
// of the rows that a tile has, those that a head with this limit sees
static_assert(tile_rows(seen_tokens(INT_MIN), 48, 16) <= 0 && tile_rows(seen_tokens(50), 48, 16) == 2 && tile_rows(INT_MAX, 48, 5) == 5, "");
"""


def test_limits_far_below_zero(tmp_path):
    """The attention kernels' arithmetic on limits, as constant expressions: one that overflows does not compile."""
    src = tmp_path / "limits.cpp"
    src.write_text(LIMITS)
    include = os.path.join(ROOT, "paper_2605_27646_amd", "csrc")
    res = subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-I", include, str(src)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    source = open(os.path.join(include, "hqmq_attend.hip")).read()
    assert source.count("a.visible[") == source.count("vis = seen_tokens(vis)") == 2


def _with(enc, **kw):
    return hq.EncodedBuffers(**{**{n: getattr(enc, n) for n in ("codes", "sigma", "flags", "row_off", "outliers", "n_outliers", "status")}, **kw})


def test_prefixes_of_short_buffers_are_refused():
    """Every part that attention and weights read is looked at: fewer rows than params says, parts that only look long enough, a
    list that has fewer bytes than payloads."""
    p, fewer = _params(), _params(T=900, stride_b=4 * 900 * 128, stride_h=900 * 128)
    full, short = hq.alloc_encoded(p, "cpu", 10), hq.alloc_encoded(fewer, "cpu", 10)
    q, out, sec = torch.zeros(6, 8, 128, dtype=torch.float16), torch.zeros(6, 8, 128, dtype=torch.float16), torch.zeros(4, 64, 4)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    bad = [short] + [_with(full, **{n: getattr(short, n)}) for n in ("codes", "sigma", "flags", "row_off")]
    bad += [_with(full, flags=full.flags[:1].expand(full.flags.shape)), _with(full, row_off=full.row_off[:-1]),
            _with(full, outliers=full.outliers[:, 0].contiguous()), _with(full, outliers=full.outliers[:, :2])]
    for e in bad:
        for k, v in ((e, full), (full, e)):
            with pytest.raises(ValueError, match="hold"):
                hq.hqmq_attend_shared(p, q, 0.1, k, sec, v, sec, out, ws)
        with pytest.raises(ValueError, match="hold"):
            hq.hqmq_attend_mass(p, q, 0.1, e, sec, torch.zeros(6, 8), torch.zeros(2, 4, 1000))
    grown = _params()
    for _ in range(2):
        assert serving._hold_rows(grown, full) is full.codes
    grown.T = 1001
    with pytest.raises(ValueError, match="hold"):
        serving._hold_rows(grown, full)


def test_params_are_as_they_were_checked():
    p = _params()
    full = hq.alloc_encoded(p, "cpu", 10)
    own = hq.OwnTokens(p, full, full)
    p.T = 5000
    assert own.params.T == 1000 and own.struct.params.contents.T == 1000


def test_windows_of_many_positions_are_taken(lib):
    """Two prompts' last 1024 positions, 32 kv heads: 65536 times B * n_share * H, which only own tokens are too many for.  (The calls
    end at a missing buffer, which is looked at later.)"""
    p = _params(B=2, H=32, T=1000, stride_b=32 * 1000 * 128)
    assert hq.hqmq_attend_shared_workspace_bytes(p, 1024, 32) > 0 and _shared(lib, params=p, n_share=1024, heads=32, ws_bytes=100) == SMALL
    own = _params(B=2048, H=32, T=10, stride_b=32 * 10 * 128, stride_h=10 * 128)
    assert hq.hqmq_attend_shared_workspace_bytes(p, 1024, 32, own) == 0
    assert _shared(lib, params=p, n_share=1024, heads=32, own=_own(own)) == UNSUPPORTED
    last = _params(B=255, H=257, T=10, stride_b=257 * 10 * 128, stride_h=10 * 128)  # 65535 heads
    assert hq.hqmq_attend_shared_workspace_bytes(last, 4, 257) > 0 and hq.hqmq_attend_shared_workspace_bytes(last, 5, 257) == 0
    for params, share, heads in ((p, 1024, 32), (last, 1024, 257 * 16)):
        assert lib.hqmq_attend_mass(C.byref(params), share, heads, P, 0.1, C.byref(_enc(sigma=0)), 5, P, P, None, P, 1.0, P, None) == INVALID


@pytest.mark.parametrize("name", ["codes", "sigma", "flags", "row_off", "outliers", "n_outliers", "status"])
def test_compact_refuses_every_buffer_of_a_given_tensor(lib, name):
    params, caps, keep = _params(), (C.c_uint64 * 2)(5, 5), (C.c_void_p * 2)(P, P)
    enc = (binding._Encoded * 2)(_enc(P), _enc(2 * P))
    at = getattr(enc[1], name)
    out = (binding._Encoded * 2)(_enc(3 * P, **{name: at}), _enc(4 * P))
    args = (C.byref(params), 10, 2, enc, caps, keep)
    assert lib.hqmq_evict_compact(*args, out, caps, P, 1 << 40, None) == INVALID
    out = (binding._Encoded * 2)(_enc(3 * P), _enc(4 * P))
    assert lib.hqmq_evict_compact(*args, out, caps, P, 16, None) == SMALL  # apart: the next check is the workspace's
