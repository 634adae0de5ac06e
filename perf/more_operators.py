"""Performance cases of prompts taken in chunks on page pools: page tables and slots of the new
tokens from the requests' lengths, rotary positions of queries and keys, compression of the new keys
and values into their slots, and attention of the chunks over the packed cache.

`run` computes them in elementary torch operations, or, with `own`, by the calls of
paper_2608_08081_amd.api.  The tokens of all sequences lie one after the other (`row_starts` says
where each begins).  Attended records are drawn directly: codes of Gaussian coordinates of variance
1/128, which is what a rotated unit vector has, and scales spread like the norms of real keys.
"""

from __future__ import annotations

import math
import random

import torch

own = False

D = 128
# positive codebook levels (Lloyd-Max on one coordinate of the unit sphere in 128 dims, in fp16)
HALF_LEVELS = (0.0216064453125, 0.06658935546875, 0.1181640625, 0.1883544921875)
# a rotated coordinate this near to a border between two codes may get either: such vectors are not
# drawn (about one in fifty)
BORDER = 4e-6
SIDES = ("k", "v")
# query heads and KV heads of draws: groups of 4 to 16, and one query head per KV head
HEADS = ((32, 4), (32, 4), (16, 2), (32, 8), (64, 8), (8, 8), (40, 8), (16, 1))
TYPES = {"fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------- the cases

def listed():
    return [
        # a decode step of a serving batch: one token each, few rows need a page
        _extend("extend_64_single_tokens", 64, 4000, 1, page=64, pages=6000),
        # a busy server's step: prompts, chunks and single tokens, the pool runs out at the end
        _extend("extend_1000_ragged", 1000, 3000, 96, page=16, pages=100000, short=True),
        # one token of a single chat, from the output of one projection: all launch and latency
        _rope("rope_1_token", 1, 32, 4, 128, "half", "fp16", far=32768, fused=True),
        # a chunk of a long document: positions around a million, pairs side by side, half a head
        _rope("rope_4099_tokens_far", 4099, 16, 2, 64, "interleaved", "fp32", far=1 << 20),
        # the prompts of a serving batch
        _rope("rope_16384_tokens", 16384, 32, 8, 128, "half", "fp16", far=65536, fused=True),
        # the new tokens of a decode batch
        _compress("compress_64_tokens", 64, 8, "fp16", page=64),
        # the prompts of a serving batch, with the padding of a captured graph
        _compress("compress_16000_tokens", 16000, 8, "fp16", page=16, pad=384),
        # the end of a short prompt: latency counts
        _attention("prefill_32_of_1000", 32, 4, [(32, 1000)], "fp16", page=16),
        # prompts, chunks and single tokens in one step, groups of 4, the padding of a graph
        _attention("prefill_mixed_20", 32, 8,
                   [(512, 8000), (300, 300), (777, 2500), (64, 9001)] + [(1, 500 * i + 77)
                                                                         for i in range(16)],
                   "fp16", page=64, pad=91),
        # layers with a window, full accuracy, groups of 5
        _attention("prefill_window_fp32", 40, 8, [(500, 6000), (1000, 1000), (129, 12345)], "fp32",
                   page=32, window=2048, sinks=4),
        # a whole prompt at once
        _attention("prefill_4096_fresh", 32, 4, [(4096, 4096)], "fp16", page=64),
        # the largest: a chunk at the end of a long context
        _attention("prefill_2048_of_32k", 32, 4, [(2048, 32768)], "fp16", page=64),
    ]


def draw(rng):
    """A case of the same ranges: 1 to 1024 sequences; 1 to 16384 new tokens to rotate and compress;
    chunks of 1 to 4096 tokens over contexts of up to 32K, windows of 64 to 8192; pages of 16 to
    64 positions, both types, both layouts."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["extend"] * 2 + ["rope"] * 2 + ["compress"] * 2 + ["prefill"] * 4)
    page = rng.choice([16, 32, 64])
    hq, hkv = rng.choice(HEADS)
    dtype = rng.choice(["fp16", "fp16", "fp32"])
    if op == "extend":
        rows = log(1, 1024)
        context, new = log(1, 4000), log(1, 512)
        pages = rows * (-(-(context + new) // page) + 1) + log(1, 2000)
        return _extend(None, rows, context, new, page=page, pages=min(pages, 150000),
                       short=rng.random() < 0.3)
    if op == "rope":
        tokens = log(1, min(16384, 16384 * 40 // (hq + hkv) // (2 if dtype == "fp32" else 1)))
        return _rope(None, tokens, hq, hkv, rng.choice([128, 128, 64, 32, 96]),
                     rng.choice(["half", "interleaved"]), dtype, far=log(1000, 1 << 21),
                     fused=rng.random() < 0.5)
    if op == "compress":
        tokens = log(1, 16384 * 8 // hkv // (2 if dtype == "fp32" else 1))
        return _compress(None, min(tokens, 16384), hkv, dtype, page=page,
                         pad=rng.choice([0, 0, 5, 128]))
    # at most the largest listed case's products
    room = 2048 * 31744 * 32 // hq
    seqs = []
    for _ in range(log(1, 32)):
        new = log(1, 4096)
        total = min(32768, new + rng.choice([0, log(1, 32768)]))
        new = min(new, total)
        if new * total <= room:
            room -= new * total
            seqs.append((new, total))
    kw = {}
    if rng.random() < 0.3:
        kw = {"window": log(64, 8192), "sinks": rng.choice([0, 1, 4, 16, 60])}
    # (the accurate form does twice the products)
    if dtype == "fp32" and room < 2048 * 31744 * 16 // hq:
        dtype = "fp16"
    return _attention(None, hq, hkv, seqs or [(1, 1000)], dtype, page=page,
                      pad=rng.choice([0, 0, 1, 64]), **kw)


def _extend(name, rows, context, new, page, pages, short=False):
    return _named({"op": "extend", "rows": rows, "context": context, "new": new, "page": page,
                   "pages": pages, "max_pages": -(-(context + 8 * new) // page) + 1,
                   "short": bool(short)}, name)


def _rope(name, tokens, q_heads, kv_heads, rope_dim, layout, dtype, far, fused=False):
    return _named({"op": "rope", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
                   "rope_dim": rope_dim, "layout": layout, "dtype": dtype, "far": far,
                   "fused": bool(fused)}, name)


def _compress(name, tokens, kv_heads, dtype, page, pad=0):
    return _named({"op": "compress", "tokens": tokens, "kv_heads": kv_heads, "dtype": dtype,
                   "page": page, "pad": pad}, name)


def _attention(name, q_heads, kv_heads, seqs, dtype, page, window=0, sinks=0, pad=0):
    # (sequences as text: new tokens, length with them)
    return _named({"op": "prefill", "q_heads": q_heads, "kv_heads": kv_heads,
                   "seqs": " ".join(f"{n}/{t}" for n, t in seqs), "dtype": dtype, "page": page,
                   "window": window, "sinks": sinks, "pad": pad}, name)


def _named(c, name):
    if name is not None:
        c["name"] = name
    return c


def _seqs(case):
    return [tuple(int(x) for x in s.split("/")) for s in case["seqs"].split()]


# --------------------------------------------------------------------------------- the inputs

def _device():
    return torch.device("cuda:0" if torch.cuda.is_available() else "cpu")


def _levels(dtype, dev):
    h = torch.tensor(HALF_LEVELS, dtype=torch.float64, device=dev)
    return torch.cat((-h.flip(0), h)).to(dtype)


def _borders(dtype, dev):
    lv = _levels(dtype, dev)
    return 0.5 * (lv[1:] + lv[:-1])


def _pack(codes):
    """codes [..][128] (int32) to records [..][48] uint8, code i at bits 3 i .. 3 i + 2."""
    sh = torch.arange(8, device=codes.device, dtype=torch.int32) * 3
    word = (codes.unflatten(-1, (16, 8)) << sh).sum(-1, dtype=torch.int32)
    by = torch.arange(3, device=codes.device, dtype=torch.int32) * 8
    return ((word.unsqueeze(-1) >> by) & 0xFF).to(torch.uint8).flatten(-2)


def _side(gen, shape, dev):
    """Records [*shape][48] and scales [*shape] of one cache side."""
    n = math.prod(shape)
    thr = _borders(torch.float32, dev)
    rec = torch.empty((n, 48), dtype=torch.uint8, device=dev)
    for i in range(0, n, 1 << 18):
        m = min(1 << 18, n - i)
        y = torch.randn((m, D), generator=gen, device=dev) * (D ** -0.5)
        rec[i:i + m] = _pack(torch.bucketize(y, thr, out_int32=True, right=True))
    norms = torch.exp(0.35 * torch.randn(n, generator=gen, device=dev)) * 14.0
    return rec.view(*shape, 48), norms.view(*shape)


def _quats(gen, heads, dev):
    q = torch.randn((heads, 32, 2, 4), generator=gen, device=dev, dtype=torch.float64)
    return (q / q.norm(dim=-1, keepdim=True)).float()


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    r = random.Random(seed * 7919 + 17)
    s = {"case": case}
    {"extend": _extend_state, "rope": _rope_state, "compress": _compress_state,
     "prefill": _prefill_state}[case["op"]](s, case, gen, r, dev)
    return s


def _int32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _extend_state(s, case, gen, r, dev):
    rows, page, n_pages, width = case["rows"], case["page"], case["pages"], case["max_pages"]
    order = list(range(n_pages))
    r.shuffle(order)
    # prompts, chunks, single tokens, and rows that wait: the same ones for every seed, in any order
    fixed = random.Random(rows)
    new = [1 if case["new"] == 1 else
           fixed.choice([0, 1, 1, fixed.randint(1, case["new"]), fixed.randint(1, 4 * case["new"])])
           for _ in range(rows)]
    r.shuffle(new)
    lens, tables, refs = [], [], [0] * n_pages
    need = 0
    for t in new:
        n = r.randint(0, case["context"])
        k = -(-n // page)
        if k > len(order) // 2:
            n = k = 0
        row = [order.pop() for _ in range(k)]
        for p in row:
            refs[p] = 1
        lens.append(n)
        need += -(-(n + t) // page) - k
        tables.append(row + [-1] * (width - k))
    # held by a cache of prompts: an eighth, or (a pool that runs out) all but nine tenths of what
    # the rows need
    held = len(order) // 8
    if case["short"]:
        held = max(held, len(order) - need * 9 // 10)
    for p in order[:held]:
        refs[p] += 1
    s["tables"], s["refs"] = _int32(tables, dev), _int32(refs, dev)
    s["lens"], s["new"] = _int32(lens, dev), _int32(new, dev)
    s["tokens"] = sum(new) + 13          # the size of the step's token arrays
    s["out_tables"], s["out_refs"] = torch.empty_like(s["tables"]), torch.empty_like(s["refs"])
    s["out_lens"] = torch.empty_like(s["lens"])
    s["row_starts"] = torch.empty(rows + 1, dtype=torch.int32, device=dev)
    s["slots"] = torch.empty(s["tokens"], dtype=torch.int64, device=dev)
    s["positions"] = torch.empty(s["tokens"], dtype=torch.int32, device=dev)
    s["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    if own:
        from paper_2608_08081_amd import api
        s["workspace"] = torch.empty(api.iq_extend_workspace_bytes(n_pages, rows),
                                     dtype=torch.uint8, device=dev)


def _rope_state(s, case, gen, r, dev):
    n, hq, hkv = case["tokens"], case["q_heads"], case["kv_heads"]
    heads = hq + 2 * hkv
    x = torch.randn((n, heads, D), generator=gen, device=dev).to(TYPES[case["dtype"]])
    s["q"], s["k"] = x[:, :hq], x[:, hq:hq + hkv]
    if not case["fused"]:
        s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
    # chunks of a few sequences, each at its own place
    pos = []
    while len(pos) < n:
        m = min(n - len(pos), r.randint(1, max(1, n // 3)))
        first = r.randint(0, max(0, case["far"] - m))
        pos += range(first, first + m)
    s["positions"] = _int32(pos, dev)
    i = torch.arange(case["rope_dim"] // 2, dtype=torch.float64, device=dev)
    s["freqs"] = 10000.0 ** (-2 * i / case["rope_dim"])
    s["q_out"] = torch.empty((n, hq, D), dtype=x.dtype, device=dev)
    s["k_out"] = torch.empty((n, hkv, D), dtype=x.dtype, device=dev)


def _compress_state(s, case, gen, r, dev):
    n, h, page = case["tokens"], case["kv_heads"], case["page"]
    total, dtype = n + case["pad"], TYPES[case["dtype"]]
    s["quats"] = _quats(gen, h, dev)
    rot, thr = _matrices(s["quats"]), _borders(torch.float64, dev)
    for side in SIDES:
        x = torch.zeros((total, h, D), dtype=dtype, device=dev)
        for g in range(h):
            have = 0
            while have < n:
                m = (n - have) * 17 // 16 + 64
                # channels of unequal scale, some of them far above the others
                scale = torch.exp(0.5 * torch.randn(D, generator=gen, device=dev))
                scale[torch.randint(D, (4,), generator=gen, device=dev)] *= 20.0
                v = (torch.randn((m, D), generator=gen, device=dev) * scale).to(dtype)
                y = v.double() @ rot[g].T.contiguous()
                y = y / v.double().norm(dim=-1, keepdim=True)
                near = (y.unsqueeze(-1) - thr).abs().amin((1, 2)) < BORDER
                v = v[~near][:n - have]
                x[have:have + len(v), g] = v
                have += len(v)
        s[side] = x
    # sequences of about a hundred tokens, from somewhere in their page on, pages in no order
    slots, n_pages = [], -(-n // page) + 2 * (n // 64 + 2)
    order = list(range(n_pages))
    r.shuffle(order)
    while len(slots) < n:
        m, at = min(n - len(slots), r.randint(64, 200)), r.randrange(page)
        pages = [order.pop() for _ in range(-(-(at + m) // page))]
        slots += [pages[(at + i) // page] * page + (at + i) % page for i in range(m)]
    s["slots"] = torch.tensor(slots + [-1] * case["pad"], dtype=torch.int64, device=dev)
    s["pool"] = {}
    for side in SIDES:
        s["pool"][side + "_codes"] = torch.zeros((n_pages, h, page, 48), dtype=torch.uint8,
                                                 device=dev)
        s["pool"][side + "_norms"] = torch.zeros((n_pages, h, page), device=dev)
    _plain_parts(s, dev)


def _prefill_state(s, case, gen, r, dev):
    seqs, page, hq, hkv = _seqs(case), case["page"], case["q_heads"], case["kv_heads"]
    n = sum(x for x, _ in seqs)
    width = -(-max(t for _, t in seqs) // page) + 1
    used = [-(-t // page) for _, t in seqs]
    n_pages = sum(used) + 3
    order = list(range(n_pages))
    r.shuffle(order)
    s["tables"] = _int32([[order.pop() for _ in range(u)] + [-1] * (width - u) for u in used], dev)
    s["lens"] = _int32([t for _, t in seqs], dev)
    starts = [0]
    for x, _ in seqs:
        starts.append(starts[-1] + x)
    s["row_starts"] = _int32(starts, dev)
    s["seqs"] = seqs
    s["cache"] = {}
    for side in SIDES:
        s["cache"][side + "_codes"], s["cache"][side + "_norms"] = _side(
            gen, (n_pages, hkv, page), dev)
    s["quats"] = _quats(gen, hkv, dev)
    s["q"] = torch.randn((n + case["pad"], hq, D), generator=gen, device=dev).to(
        TYPES[case["dtype"]])
    s["out"] = torch.zeros_like(s["q"])
    _plain_parts(s, dev)
    if own:
        from paper_2608_08081_amd import api
        s["workspace"] = torch.empty(
            api.iq_prefill_workspace_bytes(len(seqs), n + case["pad"], hq, hkv, width * page),
            dtype=torch.uint8, device=dev)


def _plain_parts(s, dev):
    """What the plain form keeps: the levels, H_128 / sqrt(128), and the signs of a conjugate."""
    s["levels"] = _levels(torch.float32, dev)
    s["hadamard"] = _hadamard(torch.float32, dev) * (D ** -0.5)
    s["conj"] = torch.tensor([1.0, -1.0, -1.0, -1.0], device=dev)


# ----------------------------------------------------------------------------------- the call

def run(s):
    if own:
        return _own(s)
    return {"extend": _plain_extend, "rope": _plain_rope, "compress": _plain_compress,
            "prefill": _plain_prefill}[s["case"]["op"]](s)


def _own(s):
    from paper_2608_08081_amd import api
    case = s["case"]
    op = case["op"]
    if op == "extend":
        api.iq_extend_pages(s["tables"], s["lens"], s["new"], s["refs"], case["page"],
                            s["row_starts"], s["slots"], s["positions"],
                            out_tables=s["out_tables"], out_lens=s["out_lens"],
                            out_refs=s["out_refs"], workspace=s["workspace"], status=s["status"])
        return _extended(s)
    if op == "rope":
        api.iq_rotate_positions(s["q"], s["k"], s["positions"], s["freqs"], layout=case["layout"],
                                q_out=s["q_out"], k_out=s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "compress":
        api.iq_compress_kv_slots(s["k"], s["v"], s["quats"], s["pool"], s["slots"])
        return s["pool"]
    out = api.iq_prefill_attention_paged(s["q"], s["cache"], s["tables"], s["row_starts"],
                                         s["lens"], s["quats"], window=case["window"],
                                         n_sinks=case["sinks"], out=s["out"],
                                         workspace=s["workspace"])
    return {"out": out}


def _extended(s):
    return {"tables": s["out_tables"], "lens": s["out_lens"], "refs": s["out_refs"],
            "row_starts": s["row_starts"], "slots": s["slots"], "positions": s["positions"],
            "status": s["status"]}


# ---------------------------------------------------------------------------- the plain forms

def _plain_extend(s):
    case = s["case"]
    page, width, tokens = case["page"], case["max_pages"], s["tokens"]
    lens, new, tables = s["lens"].long(), s["new"].long(), s["tables"]
    dev = lens.device
    total = lens + new
    starts = torch.cat((new.new_zeros(1), new.cumsum(0)))
    k = torch.arange(width, device=dev)
    # the pages that the new positions lie on, those without one fresh
    wants = (k >= (lens // page).unsqueeze(1)) & (k < (-(-total // page)).unsqueeze(1))
    wants &= (new > 0).unsqueeze(1) & (tables < 0)
    fits = total <= width * page
    wants &= fits.unsqueeze(1)
    free = torch.nonzero(s["refs"] <= 0)[:, 0]
    count = wants.sum(1)
    upto = count.cumsum(0)
    fits &= (count == 0) | (upto <= len(free))
    fresh = wants & fits.unsqueeze(1)
    rank = (fresh.flatten().cumsum(0) - 1).view(fresh.shape)
    padded = torch.cat((free, free.new_zeros(1)))
    s["out_tables"].copy_(torch.where(fresh, padded[rank.clamp(0, len(free))].int(), tables))
    s["out_refs"].copy_(s["refs"].index_put((padded[rank[fresh]],), s["refs"].new_ones(())))
    s["out_lens"].copy_(torch.where(fits, total, lens))
    s["row_starts"].copy_(starts)
    t = torch.arange(tokens, device=dev)
    row = torch.bucketize(t, starts[1:], right=True).clamp(max=len(lens) - 1)
    at = lens[row] + t - starts[row]
    there = t < starts[-1]
    entry = s["out_tables"][row, (at // page).clamp(max=width - 1)].long()
    s["positions"].copy_(torch.where(there, at, 0))
    s["slots"].copy_(torch.where(there & fits[row] & (entry >= 0), entry * page + at % page, -1))
    s["status"] |= torch.where(fits.all(), 0, 5).int()
    return _extended(s)


def _plain_rope(s):
    case = s["case"]
    m = case["rope_dim"]
    angle = s["positions"].double().unsqueeze(1) * s["freqs"]
    c, sn = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    for x, out in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
        y = x.float()
        if case["layout"] == "half":
            a, b = y[..., :m // 2], y[..., m // 2:m]
            turned = torch.cat((a * c - b * sn, a * sn + b * c), -1)
        else:
            a, b = y[..., 0:m:2], y[..., 1:m:2]
            turned = torch.stack((a * c - b * sn, a * sn + b * c), -1).flatten(-2)
        out.copy_(torch.cat((turned, y[..., m:]), -1))
    return {"q": s["q_out"], "k": s["k_out"]}


def _bit_count(x, n):
    return ((x.unsqueeze(-1) >> torch.arange(n, device=x.device)) & 1).sum(-1)


def _quat_mul(a, b):
    w, x, y, z = a.unbind(-1)
    p, q, r, t = b.unbind(-1)
    return torch.stack((w * p - x * q - y * r - z * t, w * q + x * p + y * t - z * r,
                        w * r - x * t + y * p + z * q, w * t + x * r - y * q + z * p), -1)


def _hadamard(dtype, dev):
    i = torch.arange(D, device=dev)
    return (1.0 - 2.0 * (_bit_count(i.unsqueeze(0) & i.unsqueeze(1), 7) & 1)).to(dtype)


def _forward(s, x):
    """x [..][heads][128] rotated: R x of the head."""
    ql, qr = s["quats"][:, :, 0], s["quats"][:, :, 1]
    x = (x @ s["hadamard"]).unflatten(-1, (32, 4))
    return _quat_mul(_quat_mul(ql, x), qr * s["conj"]).flatten(-2)


def _plain_compress(s):
    page = s["case"]["page"]
    keep = s["slots"] >= 0
    at = s["slots"][keep]
    for side in SIDES:
        x = s[side][keep].float()
        norm = x.double().square().sum(-1).sqrt()
        y = _forward(s, x).double() / norm.unsqueeze(-1)
        codes = torch.bucketize(y, _borders(torch.float64, y.device), out_int32=True, right=True)
        s["pool"][side + "_codes"][at // page, :, at % page] = _pack(codes)
        s["pool"][side + "_norms"][at // page, :, at % page] = norm.float()
    return s["pool"]


def _codes(records):
    """Codes [..][128] of records [..][48]."""
    dev = records.device
    by = torch.arange(3, device=dev, dtype=torch.int32) * 8
    sh = torch.arange(8, device=dev, dtype=torch.int32) * 3
    word = (records.unflatten(-1, (16, 3)).int() << by).sum(-1, dtype=torch.int32)
    return ((word.unsqueeze(-1) >> sh) & 7).flatten(-2)


def _sees(case, new, total, group, dev):
    """[new][1][total]: which positions the tokens see."""
    p = torch.arange(total - new, total, device=dev).unsqueeze(1)
    j = torch.arange(total, device=dev).unsqueeze(0)
    see = j <= p
    if case["window"]:
        see &= (j > p - case["window"]) | (j < case["sinks"])
    return see.unsqueeze(1).expand(new, group, total).flatten(0, 1)


def _plain_prefill(s):
    case = s["case"]
    page, hq, hkv = case["page"], case["q_heads"], case["kv_heads"]
    group = hq // hkv
    ql, qr, conj = s["quats"][:, None, :, 0], s["quats"][:, None, :, 1], s["conj"]
    at = 0
    for i, (new, total) in enumerate(s["seqs"]):
        # rows (token, head of the group) of each KV head
        q = s["q"][at:at + new].float().view(new, hkv, group, D).permute(0, 2, 1, 3)
        x = _forward(s, q).permute(2, 0, 1, 3).reshape(hkv, new * group, D)
        j = torch.arange(total, device=q.device)
        pages = s["tables"][i].long()[j // page]
        kv = [(s["levels"][_codes(s["cache"][side + "_codes"][pages, :, j % page])]
               * s["cache"][side + "_norms"][pages, :, j % page].unsqueeze(-1)).transpose(0, 1)
              for side in SIDES]
        a = (x @ kv[0].transpose(1, 2).contiguous()) * (D ** -0.5)
        a = a.masked_fill_(~_sees(case, new, total, group, q.device), -math.inf)
        a = a.sub_(a.amax(-1, keepdim=True)).exp_()
        o = (a @ kv[1].contiguous()) / a.sum(-1, keepdim=True)
        o = _quat_mul(_quat_mul(ql * conj, o.unflatten(-1, (32, 4))), qr).flatten(-2)
        o = (o @ s["hadamard"]).view(hkv, new, group, D).permute(1, 0, 2, 3)
        s["out"][at:at + new] = o.reshape(new, hq, D)
        at += new
    return {"out": s["out"]}


# ------------------------------------------------------------------- the work and the results

def work(case):
    """Inputs read once and outputs written once; two multiply-adds of 128 terms per seen record
    and query head."""
    size = 2 if case.get("dtype") == "fp16" else 4
    if case["op"] == "extend":
        # (the mean of the new tokens: see _extend_state)
        new = 1 if case["new"] == 1 else (2 + 2.5 * case["new"]) / 5
        return {"bytes": 8 * case["rows"] * case["max_pages"] + 8 * case["pages"]
                + 16 * case["rows"] + 12 * case["rows"] * new, "flops": 0}
    if case["op"] == "rope":
        heads = case["q_heads"] + case["kv_heads"]
        return {"bytes": case["tokens"] * (2 * heads * D * size + 4) + 4 * case["rope_dim"],
                "flops": 3 * case["tokens"] * heads * case["rope_dim"]}
    if case["op"] == "compress":
        vectors = 2 * case["tokens"] * case["kv_heads"]
        # (a butterfly of 7 sums, a block of 4 products, 7 comparisons per coordinate)
        return {"bytes": vectors * (D * size + 52) + 8 * case["tokens"] + case["kv_heads"] * 1024,
                "flops": vectors * D * 22}
    seen = pairs = tokens = 0
    for new, total in _seqs(case):
        w = case["window"] or total
        full = max(0, min(new, total - w))           # tokens whose window lies in the row
        short = new - full
        pairs += full * (w + min(case["sinks"], total)) + short * (2 * min(total, w) - short + 1) / 2
        seen += min(total, w + new + case["sinks"])
        tokens += new
    hq, hkv = case["q_heads"], case["kv_heads"]
    return {"bytes": seen * hkv * 104 + tokens * hq * D * 2 * size + hkv * 1024,
            "flops": 4 * pairs * hq * D}


def _matrices(quats):
    """[H][128][128] in 64 bits: R = diag(M_i) H_128 / sqrt(128), M_i v = q_L v conj(q_R)."""
    w, x, y, z = quats.double()[:, :, 0].unbind(-1)
    left = torch.stack((w, -x, -y, -z, x, w, -z, y, y, z, w, -x, z, -y, x, w), -1)
    w, x, y, z = quats.double()[:, :, 1].unbind(-1)
    right = torch.stack((w, x, y, z, -x, w, -z, y, -y, z, w, -x, -z, -y, x, w), -1)
    m = left.unflatten(-1, (4, 4)) @ right.unflatten(-1, (4, 4))
    two = torch.tensor([[1.0, 1.0], [1.0, -1.0]], dtype=torch.float64, device=quats.device)
    h = torch.ones((1, 1), dtype=torch.float64, device=quats.device)
    for _ in range(7):
        h = torch.kron(two, h)
    return torch.stack([torch.block_diag(*x) @ h * (D ** -0.5) for x in m])


def exact(case, seed):
    """Rotations by complex products, codes from the rotation matrices, and attention on keys and
    values taken back to the original space, all in 64 bits; page tables are whole numbers."""
    if case["op"] == "extend":
        return None
    s = prepare(case, seed)
    return {"rope": _exact_rope, "compress": _exact_compress, "prefill": _exact_prefill}[
        case["op"]](s, case)


def _exact_rope(s, case):
    m, out = case["rope_dim"], {}
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=s["q"].device),
                       s["positions"].double().unsqueeze(1) * s["freqs"]).unsqueeze(1)
    for name in ("q", "k"):
        x = s[name].double()
        if case["layout"] == "half":
            pairs = x[..., :m].unflatten(-1, (2, m // 2)).transpose(-1, -2)
        else:
            pairs = x[..., :m].unflatten(-1, (m // 2, 2))
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y = y.transpose(-1, -2) if case["layout"] == "half" else y
        x[..., :m] = y.flatten(-2)
        out[name] = x
    return out


def _exact_compress(s, case):
    rot, lv = _matrices(s["quats"]), _levels(torch.float64, s["k"].device)
    page, out = case["page"], {}
    for side in SIDES:
        codes = s["pool"][side + "_codes"].clone()
        norms = s["pool"][side + "_norms"].double()
        x = s[side][:case["tokens"]].double()
        at = s["slots"][:case["tokens"]]
        norm = x.norm(dim=-1)
        norms[at // page, :, at % page] = norm
        for g in range(case["kv_heads"]):
            y = x[:, g] @ rot[g].T.contiguous() / norm[:, g:g + 1]
            # the nearest level's index, bit by bit into its record
            code = (y.unsqueeze(-1) - lv).abs().argmin(-1)
            bits = ((code.unsqueeze(-1) >> torch.arange(3, device=y.device)) & 1).flatten(-2)
            weight = 1 << torch.arange(8, device=y.device)
            codes[at // page, g, at % page] = (bits.view(-1, 48, 8) * weight).sum(-1).to(
                torch.uint8)
        out[side + "_codes"], out[side + "_norms"] = codes, norms
    return out


def _exact_prefill(s, case):
    rot, lv = _matrices(s["quats"]), _levels(torch.float64, s["q"].device)
    hq, hkv = case["q_heads"], case["kv_heads"]
    group = hq // hkv
    out = torch.zeros_like(s["q"], dtype=torch.float64)
    at = 0
    for i, (new, total) in enumerate(s["seqs"]):
        pages = s["tables"][i, :-(-total // case["page"])].long()
        hidden = ~_sees(case, new, total, group, out.device)
        for g in range(hkv):
            kv = []
            for side in SIDES:
                rec = s["cache"][side + "_codes"][pages, g].flatten(0, 1)[:total]
                nrm = s["cache"][side + "_norms"][pages, g].flatten()[:total]
                b = (rec.unsqueeze(-1) >> torch.arange(8, device=rec.device)) & 1
                weight = torch.tensor([1, 2, 4], device=rec.device)
                code = (b.reshape(-1, D, 3).long() * weight).sum(-1)
                kv.append((lv[code] * nrm.double().unsqueeze(-1)) @ rot[g])
            hs = slice(g * group, (g + 1) * group)
            q = s["q"][at:at + new, hs].double().reshape(new * group, D)
            a = q @ kv[0].T.contiguous() * (D ** -0.5)
            a = torch.softmax(a.masked_fill_(hidden, -math.inf), -1)
            out[at:at + new, hs] = (a @ kv[1]).view(new, group, D)
        at += new
    return {"out": out}
