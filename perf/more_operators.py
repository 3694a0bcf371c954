"""Timed cases of the operators on a paged cache that is held in 4 bits and grows token by token.

  write   new K and V rows of a ragged batch are quantised into their sequences' pages and come back as the values that later
          steps will read (what attention over the new rows themselves uses): 1 to 16384 rows a call
  read    whole sequences read back from their pages: 1 to 65536 tokens
  attend  causal attention over the pages: generation steps, drafts of a few tokens, chunks of prompts; grouped queries of 1 to
          16 heads a kv head, 1 to 65536 tokens, sliding windows

Two formats, both with groups of 32 channels of a token: "float" (sign, 2 bits of exponent, 1 of mantissa, and a power of two for
the group, one byte) and "int" (0 to 15, and an fp16 scale and minimum for the group).  A page holds a power of two of tokens,
16 or more:
  k_codes   [page][head][token][width / 2]: channel 2 i in the low half of byte i, 2 i + 1 in the high half
  k_scales  [page][head][token][group][1 or 4 bytes]
  v_codes   [page][head][token / 4][width / 2 * 4]: the width in parts of 128, 64 or 32 channels (largest first); a part is
            [16][token % 4][4, 2 or 1 bytes], the 16 being consecutive runs of 8, 4 or 2 channels
  v_scales  [page][head][token / 4][group][token % 4][1 or 4 bytes]
with width the head dimension rounded up to 32, above 128 to 64.  The plain form computes in fp32.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LARGEST = 49152.0  # 6 * 2^13
MOST_PAIRS = 2 * 1024 * 16000 * 32 * 128  # query rows x tokens x heads x channels of the largest listed case
MOST_ELEMS = 64 * 8192 * 8 * 128  # of a K or V cache


def listed():
    return [
        # a generation step of eight sequences: the one new token of each, bound by launches
        {"name": "write_step", "op": "write", "n": 8, "rows": 1, "T": 1000, "ragged": False, "H": 8, "D": 128, "page": 16, "fmt": "float",
         "dtype": "fp16", "law": "normal"},
        # the prompts of four requests as they are processed together, the largest of 4096 tokens
        {"name": "write_prompts", "op": "write", "n": 4, "rows": 4096, "T": 4096, "ragged": True, "H": 8, "D": 128, "page": 64, "fmt": "float",
         "dtype": "bf16", "law": "hot"},
        # an odd batch of chunks with heads of 100 channels, of sequences that already have tokens
        {"name": "write_odd", "op": "write", "n": 7, "rows": 333, "T": 1537, "ragged": True, "H": 5, "D": 100, "page": 16, "fmt": "int",
         "dtype": "fp16", "law": "hot"},
        # a short conversation read back
        {"name": "read_short", "op": "read", "n": 1, "T": 777, "ragged": False, "H": 8, "D": 128, "page": 16, "fmt": "int", "dtype": "fp16",
         "law": "normal"},
        # two documents of 32k tokens read back, for a model with heads of 96 channels
        {"name": "read_long", "op": "read", "n": 2, "T": 32768, "ragged": False, "H": 8, "D": 96, "page": 128, "fmt": "float", "dtype": "bf16",
         "law": "normal"},
        # one conversation that has just begun: the smallest call
        {"name": "attend_short", "op": "attend", "n": 1, "rows": 1, "T": 130, "ragged": False, "H": 8, "G": 4, "D": 128, "page": 16,
         "fmt": "float", "dtype": "fp16", "law": "normal", "window": 0},
        # a generation step over a document of 32k tokens
        {"name": "attend_32k", "op": "attend", "n": 1, "rows": 1, "T": 32768, "ragged": False, "H": 8, "G": 4, "D": 128, "page": 64,
         "fmt": "float", "dtype": "fp16", "law": "hot", "window": 0},
        # a generation step of 64 sequences of up to 8k tokens: the most bytes
        {"name": "attend_batch", "op": "attend", "n": 64, "rows": 1, "T": 8192, "ragged": True, "H": 8, "G": 4, "D": 128, "page": 16,
         "fmt": "float", "dtype": "bf16", "law": "normal", "window": 0},
        # sixteen sequences of a multi-head model with heads of 64 channels, integers with minimum
        {"name": "attend_mha", "op": "attend", "n": 16, "rows": 1, "T": 2049, "ragged": True, "H": 32, "G": 1, "D": 64, "page": 32,
         "fmt": "int", "dtype": "fp16", "law": "hot", "window": 0},
        # a draft of five tokens of each of six sequences, a sliding window, heads of 96 channels
        {"name": "attend_draft", "op": "attend", "n": 6, "rows": 5, "T": 12345, "ragged": True, "H": 4, "G": 8, "D": 96, "page": 16,
         "fmt": "int", "dtype": "bf16", "law": "normal", "window": 4096},
        # the next 1024 tokens of two long prompts: the most arithmetic
        {"name": "attend_chunk", "op": "attend", "n": 2, "rows": 1024, "T": 16000, "ragged": False, "H": 8, "G": 4, "D": 128, "page": 64,
         "fmt": "float", "dtype": "bf16", "law": "hot", "window": 0},
        # a ragged batch of whole prompts with heads of 256 channels
        {"name": "attend_prompts", "op": "attend", "n": 5, "rows": 1500, "T": 1500, "ragged": True, "H": 2, "G": 4, "D": 256, "page": 32,
         "fmt": "float", "dtype": "fp16", "law": "normal", "window": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) if hi > lo else lo


def draw(rng):
    c = {"op": rng.choice(["write", "read", "attend", "attend", "attend"])}
    c["H"] = rng.choice([1, 2, 4, 8, 8, 8, 16, 32])
    c["D"] = rng.choice([128, 128, 128, 96, 64, 256, rng.randint(33, 255)])
    c["page"] = rng.choice([16, 16, 32, 64, 128])
    c["fmt"] = rng.choice(["float", "int"])
    c["dtype"] = rng.choice(["fp16", "bf16"])
    c["law"] = rng.choice(["normal", "hot"])
    c["n"] = _log_int(rng, 1, 64)
    c["ragged"] = rng.random() < 0.6
    token = c["n"] * c["H"] * _width(c["D"])
    if c["op"] == "read":
        c["T"] = _log_int(rng, 1, max(1, min(65536, (2 * 32768 * 8 * 96) // token)))
        return c
    if c["op"] == "write":
        c["rows"] = rng.choice([1, _log_int(rng, 1, max(1, min(4096, (4 * 4096 * 8 * 128) // token)))])
        c["T"] = min(65536, c["rows"] + rng.choice([0, _log_int(rng, 1, 8192)]))
        return c
    c["G"] = rng.choice([1, 2, 4, 4, 8, rng.randint(1, 16)])
    c["rows"] = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 1, max(1, min(2048, MOST_PAIRS // (token * c["G"] * 2048))))])
    most = min(65536, MOST_ELEMS // token, MOST_PAIRS // (token * c["G"] * c["rows"]))
    c["T"] = _log_int(rng, c["rows"], max(c["rows"], most))
    c["window"] = rng.choice([0, 0, _log_int(rng, 1, 8192)])
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------

def _dtype(c):
    return torch.float16 if c["dtype"] == "fp16" else torch.bfloat16


def _width(D):
    return (D + 31) // 32 * 32 if D <= 128 else (D + 63) // 64 * 64


def _sizes(c):
    """Length (with the call's rows) and number of rows of every sequence: the same for every seed, but for their order."""
    rng = random.Random(f"{c['op']} {c['n']} {c['T']} {c.get('rows')}")
    lengths = [c["T"]] * c["n"]
    if c["ragged"]:
        lengths[1:] = [rng.randint(max(1, c["T"] // 8), c["T"]) for _ in lengths[1:]]
    if c["op"] == "read":
        return lengths, lengths
    rows = [min(c["rows"], length) for length in lengths]
    if c["ragged"] and c["rows"] > 1:
        rows[1:] = [rng.randint(0, most) for most in rows[1:]]
    return lengths, rows


def _plan(c, seed):
    """What a scheduler knows of the batch, on the host: lengths, numbers of rows, the sequences' pages."""
    rng = random.Random(seed)
    pairs = list(zip(*_sizes(c)))
    rng.shuffle(pairs)
    lengths, rows = (list(x) for x in zip(*pairs))
    need = [(length + c["page"] - 1) // c["page"] for length in lengths]
    free = list(range(sum(need) + 3))
    rng.shuffle(free)
    table, at = [], 0
    for k in need:
        table.append(free[at:at + k] + [0] * (max(need) - k))
        at += k
    return lengths, rows, table, len(free)


def _values(c, role, shape, gen):
    """K (role 0) or V values, fp32 [..., heads, D] of the case's type: spread over channels, hot keys have one large channel in 32."""
    H, D = shape[-2:]
    x = torch.randn(shape, generator=gen, device=DEVICE)
    gain = torch.exp(0.3 * torch.randn(H, D, generator=gen, device=DEVICE))
    if c["law"] == "hot" and role == 0:
        gain[:, 5::32] *= 6.0
    return (x * gain).to(_dtype(c)).float()


def _inputs(case, seed):
    c, gen = case, torch.Generator(device=DEVICE).manual_seed(seed)
    lengths, rows, table, n_pages = _plan(c, seed)
    W, H, D, page = _width(c["D"]), c["H"], c["D"], c["page"]
    s = {"case": c, "lengths_host": lengths, "rows_host": rows, "n_pages": n_pages,
         "lengths": torch.tensor(lengths, dtype=torch.int32, device=DEVICE),
         "table": torch.tensor(table, dtype=torch.int32, device=DEVICE),
         "starts": torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32, device=DEVICE)}
    n_rows = sum(rows)
    if c["op"] == "write":
        s["k"], s["v"] = (_values(c, role, (n_rows, H, D), gen).to(_dtype(c)) for role in range(2))
        group = 1 if c["fmt"] == "float" else 4
        size = n_pages * H * page * W
        s["cache"] = [torch.zeros(size // 2, dtype=torch.uint8, device=DEVICE), torch.zeros(size // 32 * group, dtype=torch.uint8, device=DEVICE),
                      torch.zeros(size // 2, dtype=torch.uint8, device=DEVICE), torch.zeros(size // 32 * group, dtype=torch.uint8, device=DEVICE)]
        return s
    s["cache"] = []
    for role in range(2):
        x = _values(c, role, (n_pages, page, H, D), gen).transpose(1, 2)
        codes, scales = _quantised(c["fmt"], x, W)
        s["cache"] += [(_lay_v(codes) if role else _lay_k(codes)).reshape(-1), _lay_scales(scales, role).reshape(-1)]
    if c["op"] == "attend":
        s["q"] = (1.5 * torch.randn(n_rows, H * c["G"], D, generator=gen, device=DEVICE)).to(_dtype(c))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        s["call"] = _handle(case, s)
    return s


# ---- the framework's calls -----------------------------------------------------------------------------------------

def _handle(c, s):
    import paper_2605_27646_amd as hq

    params = hq.Cache4Params(s["n_pages"], c["page"], c["H"], c["D"], hq.HQMQ_CACHE4_FLOAT if c["fmt"] == "float" else hq.HQMQ_CACHE4_INT)
    cache = hq.Cache4Buffers(*s["cache"])
    n_rows, H, D = sum(s["rows_host"]), c["H"], c["D"]
    even = len(set(s["rows_host"])) == 1
    batch = hq.Cache4Batch(s["table"], s["lengths"], None if even else s["starts"], max_rows=max(s["rows_host"]),
                           max_length=max(s["lengths_host"]))
    if c["op"] in ("write", "read"):
        out = {"k": torch.empty(n_rows, H, D, dtype=_dtype(c), device=DEVICE), "v": torch.empty(n_rows, H, D, dtype=_dtype(c), device=DEVICE)}

        def call():
            if c["op"] == "write":
                hq.hqmq_cache4_write(params, cache, batch, s["k"], s["v"])
            hq.hqmq_cache4_read(params, cache, batch, out["k"], out["v"])
            return out
        return call
    out = {"out": torch.empty_like(s["q"]), "lse": torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEVICE)}
    ws = torch.empty(max(1, hq.hqmq_cache4_attend_workspace_bytes(params, batch, n_rows, H * c["G"], window=c["window"])), dtype=torch.uint8, device=DEVICE)

    def call():
        hq.hqmq_cache4_attend(params, cache, batch, s["q"], D ** -0.5, out["out"], ws, window=c["window"], lse=out["lse"])
        return out
    return call


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _quantised(fmt, x, W):
    """Codes uint8 [..., W] and scales uint8 [..., W / 32, 1 or 4] of fp32 rows [..., D]."""
    D = x.shape[-1]
    x = x.clamp(-LARGEST, LARGEST)
    if fmt == "float":
        x = torch.nn.functional.pad(x, (0, W - D)).unflatten(-1, (-1, 32))
        top = x.abs().amax(-1)
        e = (((top.view(torch.int32) + 0x1FFFFF) >> 23) - 129).clamp(-23, 13)
        y = x * torch.exp2(-e.float()).unsqueeze(-1)
        m = y.abs()
        code = (m > 0.25).to(torch.uint8)
        for step in (m >= 0.75, m > 1.25, m >= 1.75, m > 2.5, m >= 3.5, m > 5.0):
            code += step
        code |= (y < 0).to(torch.uint8) << 3
        return code.flatten(-2), (e + 127).to(torch.uint8).unsqueeze(-1)
    low = torch.nn.functional.pad(x, (0, W - D), value=math.inf).unflatten(-1, (-1, 32)).amin(-1)
    high = torch.nn.functional.pad(x, (0, W - D), value=-math.inf).unflatten(-1, (-1, 32)).amax(-1)
    empty = low > high
    least = torch.where(empty, 0.0, low).half()
    step = torch.where(empty, 0.0, (high - low) * torch.tensor(1 / 15, dtype=torch.float32, device=DEVICE)).half()
    x = torch.nn.functional.pad(x, (0, W - D)).unflatten(-1, (-1, 32))
    s = step.double().unsqueeze(-1)
    code = torch.where(s > 0, (x.double() - least.double().unsqueeze(-1)) / s, 0.0).round().clamp(0, 15).to(torch.uint8).flatten(-2)
    code[..., D:] = 0
    return code, torch.stack([step, least], -1).view(torch.uint8)


def _parts(W):
    at, parts = 0, []
    for width in (128, 64, 32):
        while W - at >= width:
            parts.append((at, width))
            at += width
    return parts


def _lay_k(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _lay_v(codes):
    """[P, H, page, W] -> [P, H, page / 4, W / 2 * 4]"""
    P, H, page, W = codes.shape
    x = _lay_k(codes).view(P, H, page // 4, 4, W // 2)
    return torch.cat([x[..., at // 2:(at + w) // 2].unflatten(-1, (16, w // 32)).transpose(3, 4).flatten(3) for at, w in _parts(W)], -1)


def _lay_scales(scales, role):
    P, H, page, N, n = scales.shape
    return scales.view(P, H, page // 4, 4, N, n).transpose(3, 4).contiguous() if role else scales.contiguous()


def _unlaid(c, s, role, pages):
    """Codes uint8 [..., H, page, W] and scales [..., H, page, W / 32, 1 or 4] of the given pages [...]."""
    H, page, W, P = c["H"], c["page"], _width(c["D"]), s["n_pages"]
    n = 1 if c["fmt"] == "float" else 4
    codes, scales = s["cache"][2 * role].view(P, H, -1)[pages], s["cache"][2 * role + 1].view(P, H, -1)[pages]
    lead = codes.shape[:-1]
    if role:
        x, parts, at = codes.view(*lead, page // 4, 2 * W), [], 0
        for _, w in _parts(W):
            parts.append(x[..., at:at + 2 * w].unflatten(-1, (16, 4, w // 32)).transpose(-3, -2).flatten(-2))
            at += 2 * w
        codes = torch.cat(parts, -1).flatten(-3, -2)
        scales = scales.view(*lead, page // 4, W // 32, 4, n).transpose(-3, -2).flatten(-4, -3)
    else:
        codes, scales = codes.view(*lead, page, W // 2), scales.view(*lead, page, W // 32, n)
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2), scales


def _dequantised(c, codes, scales):
    """fp32 values [..., D], those that fp16 holds."""
    if c["fmt"] == "float":
        grid = torch.tensor(GRID + tuple(-g for g in GRID), device=DEVICE)
        x = grid[codes.int()].unflatten(-1, (-1, 32)) * torch.exp2(scales.float() - 127.0)
    else:
        step, least = scales.contiguous().view(torch.float16).float().split(1, -1)
        x = (least + codes.float().unflatten(-1, (-1, 32)) * step).half().float()
    return x.flatten(-2)[..., :c["D"]]


def _places(c, s):
    """Of every row: its sequence, its position, its page and its place in the page."""
    n_rows = sum(s["rows_host"])
    row = torch.arange(n_rows, device=DEVICE)
    seq = torch.searchsorted(s["starts"][1:].long(), row, right=True)
    pos = s["lengths"].long()[seq] - s["starts"].long()[seq + 1] + row
    return seq, pos, s["table"].long()[seq, pos // c["page"]], pos % c["page"]


def _plain_write(c, s):
    H, W, page, P = c["H"], _width(c["D"]), c["page"], s["n_pages"]
    _, _, pages, place = _places(c, s)
    for role, x in enumerate((s["k"], s["v"])):
        codes, scales = _quantised(c["fmt"], x.float(), W)
        laid, flat = s["cache"][2 * role], s["cache"][2 * role + 1]
        packed = _lay_k(codes)
        if role == 0:
            laid.view(P, H, page, W // 2)[pages, :, place] = packed
            flat.view(P, H, page, W // 32, -1)[pages, :, place] = scales
            continue
        view, at = laid.view(P, H, page // 4, 2 * W), 0
        for first, w in _parts(W):
            part = view[..., at:at + 2 * w].unflatten(-1, (16, 4, w // 32))
            part[pages, :, place // 4, :, place % 4] = packed[..., first // 2:(first + w) // 2].unflatten(-1, (16, w // 32))
            at += 2 * w
        flat.view(P, H, page // 4, W // 32, 4, -1)[pages, :, place // 4, :, place % 4] = scales
    return _plain_read(c, s)


def _plain_read(c, s):
    out = {}
    seq, pos, _, _ = _places(c, s)
    at = seq * (s["table"].shape[1] * c["page"]) + pos
    for role, name in enumerate("kv"):
        codes, scales = _unlaid(c, s, role, s["table"].long())  # [n, pages, H, page, ...]
        codes, scales = (x.transpose(2, 3).flatten(0, 2)[at] for x in (codes, scales))
        out[name] = _dequantised(c, codes, scales).to(_dtype(c))
    return out


def _plain_attend(c, s):
    n, H, G, D = c["n"], c["H"], c["G"], c["D"]
    seq, pos, _, _ = _places(c, s)
    most = max(s["rows_host"])
    nth = torch.arange(seq.shape[0], device=DEVICE) - s["starts"].long()[seq]
    q = torch.zeros(n, most, H, G, D, device=DEVICE)
    q[seq, nth] = s["q"].float().view(-1, H, G, D)
    at = torch.full((n, most), -1, device=DEVICE)
    at[seq, nth] = pos
    q = q.permute(0, 2, 1, 3, 4).reshape(n, H, most * G, D)
    k, v = (_dequantised(c, *_unlaid(c, s, role, s["table"].long())).transpose(1, 2).reshape(n, H, -1, D) for role in range(2))
    t = torch.arange(k.shape[2], device=DEVICE)
    unseen = t > at.unsqueeze(-1)
    if c["window"]:
        unseen |= t <= at.unsqueeze(-1) - c["window"]
    x = (D ** -0.5 * (q @ k.transpose(2, 3))).view(n, H, most, G, -1).masked_fill_(unseen.view(n, 1, most, 1, -1), -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = x.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    o = (e.view(n, H, most * G, -1) @ v).view(n, H, most, G, D) / total.clamp_min(1e-30)
    lse = (top + torch.log(total)).squeeze(-1)
    o, lse = o.permute(0, 2, 1, 3, 4)[seq, nth], lse.permute(0, 2, 1, 3)[seq, nth]
    return {"out": o.reshape(-1, H * G, D).to(_dtype(c)), "lse": lse.reshape(-1, H * G).contiguous()}


def run(state):
    c = state["case"]
    if own:
        return state["call"]()
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[c["op"]](c, state)


# ---- in 64 bits ----------------------------------------------------------------------------------------------------

def _half64(x):
    """The fp16 value nearest to fp64 numbers, rounded once (by way of fp32, rounded to odd)."""
    f = x.float()
    f = torch.where(f.abs().double() > x.abs(), (f.view(torch.int32) - 1).view(torch.float32), f)
    odd = f.view(torch.int32) | (f.double() != x).int()
    return odd.view(torch.float32).half().double()


def _sequence64(c, s, role, i):
    """fp64 [length, H, D] of sequence i, unrounded, token by token from the pages' bytes."""
    H, page, W, D = c["H"], c["page"], _width(c["D"]), c["D"]
    t = torch.arange(s["lengths_host"][i], device=DEVICE)
    base = (s["table"][i].long()[t // page].view(-1, 1) * H + torch.arange(H, device=DEVICE)) * page  # rows of the head's page
    place = (t % page).view(-1, 1, 1)
    ch = torch.arange(D, device=DEVICE)
    if role == 0:
        byte = (base.unsqueeze(-1) + place) * (W // 2) + ch // 2
        group = (base.unsqueeze(-1) + place) * (W // 32) + ch // 32
    else:
        inner = torch.zeros(D, dtype=torch.long, device=DEVICE)
        run_bytes = torch.zeros(D, dtype=torch.long, device=DEVICE)
        for first, w in _parts(W):
            mine = (ch >= first) & (ch < first + w)
            run_bytes[mine] = w // 32
            n = (ch[mine] - first) // (w // 16)
            inner[mine] = 2 * first + n * 4 * (w // 32) + (ch[mine] - first) % (w // 16) // 2
        byte = (base.unsqueeze(-1) + place // 4 * 4) * (W // 2) + inner + place % 4 * run_bytes
        group = (base.unsqueeze(-1) + place // 4 * 4) * (W // 32) + ch // 32 * 4 + place % 4
    code = s["cache"][2 * role][byte].long() >> (4 * (ch % 2)) & 15
    scales = s["cache"][2 * role + 1]
    if c["fmt"] == "float":
        low = code & 7
        mantissa = torch.where(low < 2, low.double() / 2, (1.0 + (low % 2).double() / 2) * torch.exp2((low // 2 - 1).double()))
        return mantissa * (1.0 - 2.0 * (code >> 3)) * torch.exp2(scales[group].double() - 127.0)
    pair = scales.view(torch.float16).view(-1, 2)[group].double()
    return pair[..., 1] + code * pair[..., 0]


def _nearest64(c, x):
    """fp64 [rows, H, D]: what rows come back as, group by group."""
    x, out = x.double().clamp(-LARGEST, LARGEST), torch.empty(x.shape, dtype=torch.float64, device=DEVICE)
    for first in range(0, c["D"], 32):
        g = x[..., first:first + 32]
        if c["fmt"] == "float":
            m, e = torch.frexp(g.abs().amax(-1, keepdim=True))  # m 2^e, m from 1/2 to 1: up to 7 * 2^(e - 3) if m is at most 7/8
            e = torch.where(m == 0.0, -23, torch.where(m <= 0.875, e - 3, e - 2).clamp(-23, 13))
            unit = torch.exp2(e.double())
            grid = torch.tensor(GRID, dtype=torch.float64, device=DEVICE)
            far = ((g.abs() / unit).unsqueeze(-1) - grid).abs() + 1e-9 * (torch.arange(8, device=DEVICE) % 2)  # ties: even codes
            out[..., first:first + 32] = torch.sign(g) * grid[far.argmin(-1)] * unit
            continue
        low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
        step = ((high - low).float().double() * float(torch.tensor(1 / 15, dtype=torch.float32))).float().half().double()
        least = low.float().half().double()
        code = ((g - least) / torch.where(step > 0, step, 1.0)).round().clamp(0, 15)
        out[..., first:first + 32] = least + code * step
    return out


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    H, D = c["H"], c["D"]
    if c["op"] == "write":
        return {name: _nearest64(c, s[name]) for name in "kv"}
    if c["op"] == "read":
        return {name: torch.cat([_sequence64(c, s, role, i) for i in range(c["n"])]) for role, name in enumerate("kv")}
    G = c["G"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEVICE)
    first = 0
    for i, rows in enumerate(s["rows_host"]):
        length = s["lengths_host"][i]
        k, v = (_sequence64(c, s, role, i) for role in range(2))
        if c["fmt"] == "int":
            k, v = _half64(k), _half64(v)
        p = torch.arange(length - rows, length, device=DEVICE).view(-1, 1)
        t = torch.arange(length, device=DEVICE)
        unseen = t > p
        if c["window"]:
            unseen |= t <= p - c["window"]
        for h in range(H):
            for g in range(h * G, (h + 1) * G):
                x = D ** -0.5 * (s["q"][first:first + rows, g].double() @ k[:, h].T)
                x = x.masked_fill(unseen, -math.inf)
                log = torch.logsumexp(x, -1, keepdim=True)
                out[first:first + rows, g] = torch.exp(x - log) @ v[:, h]
                lse[first:first + rows, g] = log.squeeze(-1)
        first += rows
    return {"out": out, "lse": lse}


# ---- the work that no method can leave out -------------------------------------------------------------------------

def _pairs(rows, length, window):
    """Tokens seen, summed over the last rows positions of a sequence."""
    if not window or window >= length:
        return rows * length - rows * (rows - 1) // 2
    short = max(0, min(rows, window - (length - rows) - 1))  # rows that see less than a window
    first = length - rows + 1
    return sum(range(first, first + short)) + (rows - short) * window


def work(case):
    """Rows and packed pages once.  Arithmetic: the two products, or an operation an element to move between values and codes."""
    c = case
    H, D = c["H"], c["D"]
    lengths, rows = _sizes(c)
    packed = D / 2 + (1 if c["fmt"] == "float" else 4) * D / 32  # bytes of a head's row of K or V
    if c["op"] == "read":
        return {"bytes": int(sum(rows) * H * 2 * (2 * D + packed)), "flops": sum(rows) * H * 2 * D}
    if c["op"] == "write":
        return {"bytes": int(sum(rows) * H * 2 * (4 * D + packed)), "flops": sum(rows) * H * 4 * D}
    heads = H * c["G"]
    seen = sum(_pairs(r, length, c["window"]) for r, length in zip(rows, lengths))
    reach = sum(min(length, c["window"] + r - 1 if c["window"] else length) for r, length in zip(rows, lengths) if r)
    return {"bytes": int(reach * H * 2 * packed + sum(rows) * heads * (4 * D + 4)), "flops": 4 * seen * heads * D}
