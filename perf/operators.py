"""The operators of a decode layer, measured: the paged 4-bit latent cache, the attention that reads it, 4-bit W_b.

Four kinds of call, each through the package's public entry points (`own`) or as elementary torch operations:

  append   new rows into the paged cache (latent in 4 bits, RoPE key rotated to its position), and those rows read back as
           the kv stream that the online attention takes (cache_append, cache_gather)
  attend   absorbed-MLA attention of new tokens over the paged 4-bit cache of a batch of requests, whose documents may
           lie in their own canonical frames (cache_attend)
  wb       the shared second projection y = W_b z with W_b in 4 bits (shared_wb_mx4)
  mx4      a weight into 4 bits and back (mx4_quantize, mx4_dequantize)

Widths and head counts are those of the paper's geometries (512 + 64 latent, 64 or 128 heads, or one device's share of
them).  A case fixes every size; the seed gives the values and where in the cache the rows lie.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

D_C, D_R = 512, 64
ROW_BYTES = D_C // 2 + D_C // 32 + 2 * D_R     # codes, scales, bf16 RoPE key
ROPE_BASE = 10000.0
SCALE = 1.0 / math.sqrt(192.0)
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def listed():
    return [
        # one decode step of a batch: a new row for each request, launches and latency
        dict(name="append_32", kind="append", rows=32, page_rows=64, rotate=True, stride=576),
        # documents of a prompt into the cache, in the frame they are stored in, out of a wider projection's output
        dict(name="append_33k", kind="append", rows=33792, page_rows=64, rotate=False, stride=640),
        # the smallest decode: one request after a short prompt
        dict(name="attend_1x2k", kind="attend", seqs=1, keys=2100, ragged=False, docs=5, heads=64, n_q=1, page_rows=64, pad=0, layout=1),
        # one device's share of the heads (8 devices), a batch of ordinary chats
        dict(name="attend_48x6k_16heads", kind="attend", seqs=48, keys=6000, ragged=True, docs=0, heads=16, n_q=1, page_rows=128, pad=2, layout=2),
        # a full batch over retrieved documents, all 64 heads
        dict(name="attend_64x16k", kind="attend", seqs=64, keys=16000, ragged=True, docs=8, heads=64, n_q=1, page_rows=64, pad=0, layout=3),
        # the 128-head geometry with a drafted token beside the new one
        dict(name="attend_16x8k_128heads_2q", kind="attend", seqs=16, keys=8200, ragged=True, docs=4, heads=128, n_q=2, page_rows=64, pad=1, layout=4),
        # one request over the long prompt: 64 documents of 4096 tokens and a query block
        dict(name="attend_1x264k", kind="attend", seqs=1, keys=264192, ragged=False, docs=64, heads=64, n_q=1, page_rows=64, pad=0, layout=5),
        # W_b for a single new token, for a batch, and for a wide layer and a chunk of tokens
        dict(name="wb_1", kind="wb", rows=1, d_in=4096, d_out=4096, out="f32"),
        dict(name="wb_32_wide", kind="wb", rows=32, d_in=7168, d_out=16384, out="bf16"),
        dict(name="wb_200", kind="wb", rows=200, d_in=4096, d_out=7168, out="bf16"),
        # W_b into 4 bits and back when a model is loaded: a small odd one, an ordinary one
        dict(name="mx4_512x2000", kind="mx4", rows=2000, cols=512, stride=520),
        dict(name="mx4_16384x7168", kind="mx4", rows=16384, cols=7168, stride=7168),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["append"] * 2 + ["attend"] * 5 + ["wb"] * 3 + ["mx4"])
    if kind == "append":
        return dict(kind=kind, rows=_log(rng, 1, 100000), page_rows=rng.choice([64, 128, 256]), rotate=rng.random() < 0.6,
                    stride=rng.choice([576, 576, 584, 640, 2112]))
    if kind == "wb":
        d_in, d_out = rng.choice([(4096, 4096), (7168, 4096), (4096, 7168), (2048, 1024), (512, 2000), (128, 128), (64, 3), (16384, 520)])
        return dict(kind=kind, rows=_log(rng, 1, 300), d_in=d_in, d_out=d_out + rng.choice([0, 0, 1, 5, 16]), out=rng.choice(["f32", "bf16"]))
    if kind == "mx4":
        cols = 32 * _log(rng, 1, 224)
        return dict(kind=kind, rows=_log(rng, 1, 16384), cols=cols, stride=cols + 8 * rng.randrange(3))
    seqs, keys = _log(rng, 1, 160), _log(rng, 1, 264192)
    case = dict(kind=kind, seqs=seqs, keys=keys, ragged=rng.random() < 0.8, docs=rng.choice([0, 0, 1, 3, 12]),
                heads=rng.choice([8, 16, 16, 32, 64, 64, 128, 20]), n_q=rng.choice([1, 1, 1, 2, 3, 4]),
                page_rows=rng.choice([64, 64, 128, 256]), pad=rng.choice([0, 0, 1, 3]), layout=rng.randrange(1 << 20))
    # no dearer than the full batch
    while case["seqs"] * case["keys"] > 900000 or work(case)["flops"] > 1.3e11:
        if case["seqs"] > 1:
            case["seqs"] = max(1, case["seqs"] * 2 // 3)
        else:
            case["keys"] = case["keys"] * 2 // 3
    return case


# ---------------------------------------------------------------------------
# structure of an attend case: each request's lengths and page entries
# ---------------------------------------------------------------------------
def _lengths(case):
    rng = random.Random(case["layout"])
    if not case["ragged"]:
        return [case["keys"]] * case["seqs"]
    return [max(1, min(2 * case["keys"], round(case["keys"] * rng.uniform(0.05, 1.95)))) for _ in range(case["seqs"])]


def _requests(case):
    """Per request: (segments, t of its last token), a segment = (request position, rows, frame).  Its documents, in their
    own frames and stored in any order, then the rows of its own (question and answer so far) at their positions."""
    rng = random.Random(case["layout"] + 1)
    got = []
    for n in _lengths(case):
        segs, at = [], 0
        docs = min(case["docs"], n // 2)
        if docs:
            part = n - max(1, n // 16)
            cuts = [0] + sorted(rng.randrange(0, part + 1) for _ in range(docs - 1)) + [part]
            for lo, hi in zip(cuts, cuts[1:]):
                if hi > lo:
                    segs.append((lo, hi - lo, lo))
                    at = hi
            rng.shuffle(segs)
        segs.append((at, n - at, 0))
        got.append((segs, n - 1))
    return got


def _pages(segs, page_rows):
    """Page entries of a request: (rows, request position, frame) a page; the last, own, page is open."""
    got = []
    for k, (at, rows, frame) in enumerate(segs):
        for u in range(0, rows, page_rows):
            got.append((page_rows if k == len(segs) - 1 else min(page_rows, rows - u), at + u, frame))
    return got


# ---------------------------------------------------------------------------
# 4-bit groups in plain torch
# ---------------------------------------------------------------------------
def _to_mx4(x):
    """Codes [.., n / 2] and scales [.., n / 32] (uint8) of finite values x [.., n] in groups of 32."""
    g = x.float().reshape(*x.shape[:-1], -1, 32)
    a = g.abs().amax(-1, keepdim=True)
    e = torch.frexp(a)[1] - 3                                    # floor(log2 a) - 2
    e = (e + (a >= torch.ldexp(torch.full_like(a, 7.0), e))).clamp(-127, 127)
    e = torch.where(a == 0, torch.full_like(e, -127), e)
    v = torch.ldexp(torch.ldexp(g, -(e // 2)), e // 2 - e)       # two steps: 2^-e may pass the range
    m = v.abs()
    code = torch.where(m < 2, (m * 2).round(), torch.where(m < 4, m.round() + 2, ((m / 2).round() + 4).clamp(max=7)))
    code = (code.to(torch.uint8) + 8 * torch.signbit(g).to(torch.uint8)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8).squeeze(-1)


def _from_mx4(codes, scales, dtype=torch.float32):
    """The values [.., 2 x codes] that codes and scales stand for (scale byte 255: NaN)."""
    table = torch.tensor(E2M1, dtype=dtype, device=codes.device)
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).flatten(-2)
    e = scales.to(torch.int32) - 127
    v = v.unflatten(-1, (-1, 32))
    v = torch.ldexp(torch.ldexp(v, (e // 2).unsqueeze(-1)), (e - e // 2).unsqueeze(-1))
    return torch.where((scales == 255).unsqueeze(-1), torch.full_like(v, math.nan), v).flatten(-2)


def _planes(cache, page_rows):
    """Views of the cache's codes, scales and RoPE keys, [pages, page_rows, ..]."""
    c, s = page_rows * D_C // 2, page_rows * (D_C // 2 + D_C // 32)
    return (cache[:, :c].unflatten(1, (page_rows, D_C // 2)), cache[:, c:s].unflatten(1, (page_rows, D_C // 32)),
            cache[:, s:].view(torch.bfloat16).unflatten(1, (page_rows, D_R)))


def _rotated(x, turns):
    """x [.., 64] with its pairs (j, j + 32) rotated by `turns` [..] positions; angles in 64 bits."""
    freq = ROPE_BASE ** (-torch.arange(D_R // 2, dtype=torch.float64, device=x.device) * 2 / D_R)
    a = turns.double().unsqueeze(-1) * freq
    c, s = a.cos().to(x.dtype), a.sin().to(x.dtype)
    x1, x2 = x[..., : D_R // 2], x[..., D_R // 2:]
    return torch.cat((x1 * c - x2 * s, x1 * s + x2 * c), -1)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _geom(heads):
    return SimpleNamespace(n_heads=heads, n_groups=1, d_latent=D_C, d_rope=D_R, d_model=4096, n_proj_groups=1,
                           softmax_scale=SCALE, rope_base=ROPE_BASE)


def _latents(gen, n, width):
    """Rows as a layer gives them: unit values, channels of their own size, a few large ones."""
    size = torch.exp2(torch.randn((1, width), generator=gen, device="cuda"))
    return torch.randn((n, width), generator=gen, device="cuda") * size


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "append":
        n, pr = case["rows"], case["page_rows"]
        pages = -(-n * 5 // 4 // pr) + 1
        s["kv"] = _latents(gen, n, case["stride"]).to(torch.bfloat16)[:, : D_C + D_R]
        s["pos"] = torch.randint(0, 264192, (n,), generator=gen, device="cuda", dtype=torch.int32) if case["rotate"] else None
        s["slots"] = torch.randperm(pages * pr, generator=gen, device="cuda")[:n].to(torch.int32)
        if n > 4 * pr:   # documents: whole pages in any order, rows in order
            at = torch.randperm(pages, generator=gen, device="cuda")
            s["slots"] = (at[:, None] * pr + torch.arange(pr, device="cuda")).flatten()[:n].to(torch.int32)
        s["cache"] = torch.zeros((pages, pr * ROW_BYTES), dtype=torch.uint8, device="cuda")
        s["back"] = torch.zeros((n, D_C + D_R), dtype=torch.bfloat16, device="cuda")
        s["geom"] = _geom(64)
    elif case["kind"] == "attend":
        reqs, pr, nq = _requests(case), case["page_rows"], case["n_q"]
        lists = [_pages(segs, pr) for segs, _ in reqs]
        count = [len(x) for x in lists]
        total = sum(count) + 3
        ids = torch.randperm(total, generator=gen, device="cuda").cpu().numpy()
        table = np.zeros((len(reqs), max(count), 4), dtype=np.int32)
        at = 0
        for b, x in enumerate(lists):
            table[b, : len(x), 0] = ids[at: at + len(x)]
            table[b, : len(x), 1:] = x
            at += len(x)
        table[:, :, 0] = np.where(np.arange(max(count)) < np.array(count)[:, None], table[:, :, 0], -1)   # nothing there
        t = np.array([t for _, t in reqs], dtype=np.int32)[:, None] + np.arange(1 - nq, 1, dtype=np.int32)
        if case["pad"]:   # the batch is padded to its captured size: these rows belong to no request
            t[len(reqs) - min(case["pad"], len(reqs) - 1):] = -1
        s["pages"] = torch.from_numpy(table).cuda()
        s["seq_pages"] = torch.tensor(count, dtype=torch.int32, device="cuda")
        s["pos"] = torch.from_numpy(np.ascontiguousarray(t)).cuda()
        s["cache"] = torch.zeros((total, pr * ROW_BYTES), dtype=torch.uint8, device="cuda")
        codes, scales, rope = _planes(s["cache"], pr)
        for lo in range(0, total, 1 << 12):
            hi = min(total, lo + (1 << 12))
            c, e = _to_mx4(torch.randn((hi - lo, pr, D_C), generator=gen, device="cuda").to(torch.bfloat16))
            codes[lo:hi], scales[lo:hi] = c, e
            rope[lo:hi] = torch.randn((hi - lo, pr, D_R), generator=gen, device="cuda").to(torch.bfloat16)
        # rows that were never written hold anything
        own_at = torch.from_numpy(np.array([x[-1] for x in lists])).cuda()
        page = s["pages"][torch.arange(len(reqs), device="cuda"), s["seq_pages"].long() - 1, 0].long()
        free = own_at[:, 1, None] + torch.arange(pr, device="cuda") > torch.tensor([t for _, t in reqs], device="cuda")[:, None]
        b, i = free.nonzero(as_tuple=True)
        scales[page[b], i] = 255
        s["q"] = (torch.randn((len(reqs), nq, case["heads"], D_C + D_R), generator=gen, device="cuda") * 0.5).to(torch.bfloat16)
        s["out_o"] = torch.zeros((len(reqs), nq, case["heads"], D_C), dtype=torch.bfloat16, device="cuda")
        s["out_lse"] = torch.zeros((len(reqs), nq, case["heads"]), dtype=torch.float32, device="cuda")
        s["geom"] = _geom(case["heads"])
    elif case["kind"] == "wb":
        w = torch.randn((case["d_out"], case["d_in"]), generator=gen, device="cuda") * 0.02
        s["codes"], s["scales"] = _to_mx4(w.to(torch.bfloat16))
        s["z"] = torch.randn((case["rows"], case["d_in"]), generator=gen, device="cuda").to(torch.bfloat16)
        s["y"] = torch.zeros((case["rows"], case["d_out"]), dtype=_dtype(case), device="cuda")
    else:
        n, cols = case["rows"], case["cols"]
        s["w"] = (torch.randn((n, case["stride"]), generator=gen, device="cuda") * 0.02).to(torch.bfloat16)[:, :cols]
        s["codes"] = torch.zeros((n, cols // 2), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.zeros((n, cols // 32), dtype=torch.uint8, device="cuda")
        s["back"] = torch.zeros((n, cols), dtype=torch.bfloat16, device="cuda")
    return s


def _dtype(case):
    return torch.bfloat16 if case["out"] == "bf16" else torch.float32


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attend": _attend, "wb": _wb, "mx4": _mx4}[s["case"]["kind"]](s)


def _own(s):
    from paper_2609_07008_amd import mla
    case = s["case"]
    if case["kind"] == "append":
        mla.cache_append(s["geom"], s["kv"], s["slots"], s["cache"], case["page_rows"], pos=s["pos"])
        mla.cache_gather(s["geom"], s["slots"], s["cache"], case["page_rows"], s["back"])
        return s["back"]
    if case["kind"] == "attend":
        if "ws" not in s:   # a decode loop's workspace, allocated once
            need = mla.cache_attend_query(s["geom"], case["seqs"], case["n_q"], s["pages"].shape[1], case["page_rows"])
            s["ws"] = torch.empty((max(need, 256),), dtype=torch.uint8, device="cuda")
        mla.cache_attend(s["geom"], s["q"], s["pos"], s["pages"], s["seq_pages"], s["cache"], case["page_rows"], s["out_o"],
                         s["out_lse"], workspace=s["ws"])
        return s["out_o"], s["out_lse"]
    if case["kind"] == "wb":
        mla.shared_wb_mx4(s["z"], s["codes"], s["scales"], s["y"])
        return s["y"]
    mla.mx4_quantize(s["w"], s["codes"], s["scales"])
    mla.mx4_dequantize(s["codes"], s["scales"], s["back"])
    return s["back"]


def _append(s):
    pr = s["case"]["page_rows"]
    codes, scales, rope = _planes(s["cache"], pr)
    page, row = (s["slots"] // pr).long(), (s["slots"] % pr).long()
    c, e = _to_mx4(s["kv"][:, :D_C])
    k = s["kv"][:, D_C:]
    codes[page, row], scales[page, row] = c, e
    rope[page, row] = k if s["pos"] is None else _rotated(k.float(), s["pos"]).to(torch.bfloat16)
    return torch.cat((_from_mx4(codes[page, row], scales[page, row]).to(torch.bfloat16), rope[page, row]), -1)


def _attend(s):
    pr, pages = s["case"]["page_rows"], s["pages"].long()
    codes, scales, rope = _planes(s["cache"], pr)
    nb, most = pages.shape[:2]
    i = torch.arange(pr, device="cuda")
    there = (torch.arange(most, device="cuda") < s["seq_pages"][:, None]) & (pages[..., 0] >= 0)
    ids = torch.where(there, pages[..., 0], 0)
    at = (pages[..., 2, None] + i).flatten(1)                                   # [b, keys] request positions
    kept = (there[..., None] & (i < pages[..., 1, None])).flatten(1)
    latent = _from_mx4(codes[ids], scales[ids]).flatten(1, 2)
    # keys turned from their page's frame to their positions in the request, as a cache without frames holds them
    key = _rotated(rope[ids].float(), pages[..., 3, None].expand(nb, most, pr)).flatten(1, 2)
    q = s["q"].float()
    nq, heads = q.shape[1:3]
    t = s["pos"][..., None].expand(nb, nq, heads)
    q_r = _rotated(q[..., D_C:], t).flatten(1, 2)
    seen = kept[:, None] & (at[:, None] <= t.flatten(1)[..., None])              # [b, rows, keys]
    latent = torch.where(kept[..., None] & (at <= s["pos"].amax(1, keepdim=True))[..., None], latent, 0.0)
    x = torch.matmul(q[..., :D_C].flatten(1, 2), latent.transpose(1, 2).contiguous())
    x = (x + torch.matmul(q_r, key.transpose(1, 2).contiguous())) * SCALE
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, latent) / torch.where(total == 0, 1.0, total)
    lse = (m + torch.log(total)).squeeze(-1)
    return o.to(torch.bfloat16).unflatten(1, (nq, heads)), lse.unflatten(1, (nq, heads))


def _wb(s):
    return torch.matmul(s["z"].float(), _from_mx4(s["codes"], s["scales"]).t()).to(s["y"].dtype)


def _mx4(s):
    codes, scales = _to_mx4(s["w"])
    return _from_mx4(codes, scales).to(torch.bfloat16)


def work(case):
    if case["kind"] == "append":
        n = case["rows"]
        moved = 2 * (D_C + D_R) + ROW_BYTES
        return {"bytes": n * (2 * moved + 8 + (4 if case["rotate"] else 0)), "flops": n * (2 * D_C + (6 * D_R if case["rotate"] else 0))}
    if case["kind"] == "attend":
        lens = _lengths(case)
        lens = lens[: len(lens) - min(case["pad"], len(lens) - 1)] if case["pad"] else lens
        h, nq = case["heads"], case["n_q"]
        seen = sum(max(0, n - j) for n in lens for j in range(nq))
        rows = case["seqs"] * nq * h
        return {"bytes": sum(lens) * ROW_BYTES + rows * (2 * (D_C + D_R) + 2 * D_C + 4), "flops": 2.0 * seen * h * (2 * D_C + D_R)}
    if case["kind"] == "wb":
        n, i, o = case["rows"], case["d_in"], case["d_out"]
        return {"bytes": i * o * 17 // 32 + n * (2 * i + (2 if case["out"] == "bf16" else 4) * o), "flops": 2.0 * n * i * o}
    n = case["rows"] * case["cols"]
    return {"bytes": n * (4 + 2 * 17 / 32), "flops": 4.0 * n}


# ---------------------------------------------------------------------------
# the definitions in 64 bits, one row, group or request at a time
# ---------------------------------------------------------------------------
def _group_values(x):
    """What groups [.., 32] (64 bits, finite) stand for in 4 bits: the nearest of the sixteen values times a power of two,
    found by comparing with all of them; a value halfway goes to the even code."""
    a = np.abs(x).max(-1, keepdims=True)
    e = np.floor(np.log2(np.where(a > 0, a, 1.0))) - 2
    e = np.clip(np.where(a >= 7 * 2.0 ** e, e + 1, e), -127, 127)
    levels = np.array(E2M1[:8])
    v = np.abs(x) / 2.0 ** e
    code = np.zeros(x.shape, dtype=np.int64)
    for k in range(7):
        half = (levels[k] + levels[k + 1]) / 2
        code = np.where((v > half) | ((v == half) & (k % 2 == 1)), k + 1, code)
    return np.sign(x) * levels[code] * 2.0 ** e


def _all_groups(x):
    """_group_values of [n, width] on the host, some rows at a time."""
    got = np.empty(x.shape, dtype=np.float64)
    for lo in range(0, x.shape[0], 4096):
        rows = x[lo: lo + 4096].double().cpu().numpy()
        got[lo: lo + 4096] = _group_values(rows.reshape(rows.shape[0], -1, 32)).reshape(rows.shape)
    return got


def exact(case, seed):
    if case["kind"] in ("append", "mx4") and case["rows"] * case.get("cols", D_C) > 3.0e7:
        return None
    s = prepare(case, seed)
    if case["kind"] == "append":
        k = s["kv"][:, D_C:].double().cpu().numpy()
        if case["rotate"]:
            z = (k[:, : D_R // 2] + 1j * k[:, D_R // 2:]) * np.exp(
                1j * s["pos"].cpu().numpy().astype(np.float64)[:, None] * ROPE_BASE ** (-2.0 * np.arange(D_R // 2) / D_R))
            k = np.concatenate((z.real, z.imag), 1)
        return np.concatenate((_all_groups(s["kv"][:, :D_C]), k), 1)
    if case["kind"] == "mx4":
        return _all_groups(s["w"])
    if case["kind"] == "wb":
        v = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
        byte = s["codes"].long()
        w = torch.empty((case["d_out"], case["d_in"]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = v[byte % 16], v[byte // 16]
        w *= torch.pow(2.0, s["scales"].double() - 127).repeat_interleave(32, 1)
        return s["z"].double() @ w.t()
    pr, nq, heads = case["page_rows"], case["n_q"], case["heads"]
    table, count, pos = s["pages"].cpu().numpy(), s["seq_pages"].cpu().numpy(), s["pos"].cpu().numpy()
    raw = s["cache"]
    v = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    freq = torch.pow(torch.tensor(ROPE_BASE, dtype=torch.float64), -torch.arange(0, D_R, 2, dtype=torch.float64) / D_R).cuda()
    out = torch.zeros((case["seqs"], nq, heads, D_C), dtype=torch.float64, device="cuda")
    lse = torch.full((case["seqs"], nq, heads), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        entries = table[b, : count[b]]
        data = raw[torch.from_numpy(entries[:, 0].astype(np.int64)).cuda()]
        n = entries.shape[0] * pr
        byte = data[:, : pr * 256].reshape(n, 256).long()
        c = torch.empty((n, D_C), dtype=torch.float64, device="cuda")
        c[:, 0::2], c[:, 1::2] = v[byte % 16], v[byte // 16]
        c *= torch.pow(2.0, data[:, pr * 256: pr * 272].reshape(n, 16).double() - 127).repeat_interleave(32, 1)
        k = data[:, pr * 272:].contiguous().view(torch.bfloat16).reshape(n, D_R).double()
        kz = torch.complex(k[:, : D_R // 2], k[:, D_R // 2:])
        u = torch.arange(n, device="cuda") % pr
        e = torch.from_numpy(entries.astype(np.int64)).cuda().repeat_interleave(pr, 0)
        for j in range(nq):
            t = int(pos[b, j])
            use = ((u < e[:, 1]) & (e[:, 2] + u <= t)).nonzero().squeeze(1)
            if not use.numel():
                continue
            q = s["q"][b, j].double()
            qz = torch.complex(q[:, D_C: D_C + D_R // 2], q[:, D_C + D_R // 2:])
            # each key meets the query turned into its own frame
            turned = kz[use] * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), -(t - e[use, 3, None]).double() * freq)
            x = (q[:, :D_C] @ c[use].t() + qz.real @ turned.real.t() + qz.imag @ turned.imag.t()) * SCALE
            lse[b, j] = torch.logsumexp(x, 1)
            out[b, j] = torch.softmax(x, 1) @ c[use]
    return out, lse
