"""GPU tests of prompts in chunks where they can go wrong: many rows with few beside them, rows of
zeros and of far norms, non-finite values in seen and in masked places, page entries outside the
pools, strides, streams, graphs, many sequences, pools beyond 2^32 bytes, and all operators of a
serving step together over several steps."""

import numpy as np
import pytest
import torch

from oracle import compress as ocz
from paper_2608_08081_amd import _lib, api
from tests import prefill as pf
from tests import serving as sv
from tests.test_gpu_prefill import attention_case, extend_case

pytestmark = pytest.mark.gpu
D = 128
MIXED = [(100, 400), (1, 700), (2, 90), (4, 1300), (3, 3), (0, 40)]


def attend(q, pool, tables, starts, lens, quats, **kw):
    return api.iq_prefill_attention_paged(q.to(sv.DEV), sv.as_dict(pool), sv.dev(tables),
                                          sv.dev(starts), sv.dev(lens), sv.dev(quats), **kw)


# ---- rows -------------------------------------------------------------------------------------
@pytest.mark.parametrize("window,sinks", [(0, 0), (5, 0), (40, 3), (129, 64), (900, 70)])
@pytest.mark.parametrize("seqs,hq,hkv", [(MIXED, 16, 2), ([(260, 260)], 8, 4), ([(31, 2000)], 16, 1),
                                         ([(513, 600), (1, 64), (33, 333)], 5, 1)],
                         ids=["mixed", "fresh", "end", "odd"])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_many_rows(window, sinks, seqs, hq, hkv, dtype):
    rng = np.random.default_rng([window, sinks, hq])
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, hq, hkv, 16, dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, hkv, window, sinks)
    out = attend(q, pool, tables, starts, lens, quats, window=window, n_sinks=sinks)
    pf.check_attention(out, want, dtype, f"{seqs} {window}/{sinks}")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("seqs", [[(64, 700)], [(6, 90), (1, 40)]], ids=["many", "few"])
def test_zero_nonfinite_and_far_rows(dtype, seqs):
    """A row of zeros weighs all positions alike; NaN or infinite rows stay what they are; neither
    these nor rows of a far norm cost the others of their block anything."""
    rng = np.random.default_rng(7)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 16, 2, 16, dtype)
    q = q * torch.from_numpy(np.exp(1.5 * rng.standard_normal(q.shape[:2]))).to(dtype)[..., None]
    q[1, 3] = 0
    q[2] = 0
    bad = torch.zeros(q.shape[:2], dtype=torch.bool)
    for t, h, d, x in ((0, 0, 5, float("nan")), (3, 9, 127, float("inf")), (4, 15, 0, -float("inf"))):
        q[t, h, d] = x
        bad[t, h] = True
    finite = torch.where(bad[..., None], torch.zeros_like(q), q)
    want = pf.attention(finite.double().numpy(), rows, starts, lens, quats, 2)
    out = attend(q, pool, tables, starts, lens, quats).cpu()
    assert torch.all(~torch.isfinite(out[bad])), "a non-finite row is finite"
    keep = ~bad.numpy()
    pf.check_attention(out[~bad], tuple(x[keep] for x in want), dtype, f"far rows {seqs}")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_all_rows_zero(dtype):
    rng = np.random.default_rng(8)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, [(40, 300)], 16, 2, 16, dtype)
    q.zero_()
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2)
    pf.check_attention(attend(q, pool, tables, starts, lens, quats), want, dtype, "zeros")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_large_scores(dtype):
    """Scores of hundreds, which grow along the sequence: references are raised late, and weights
    that fp16 cannot hold are made again."""
    rng = np.random.default_rng(9)
    seqs = [(80, 900), (3, 500)]
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 16, 2, 16, dtype)
    ramp = np.exp(np.linspace(-3, 3, rows[1].shape[2])).astype(np.float32)
    rows[1] = rows[1] * ramp
    pool, tables = sv.to_pool(rng, rows, lens, 16, tables.shape[1])
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2)
    assert want[1].max() > 200
    pf.check_attention(attend(q, pool, tables, starts, lens, quats), want, dtype, "large scores")


# ---- scales that are not finite, or far apart -------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("seqs", [[(300, 900), (40, 100)], [(12, 900), (9, 100)]], ids=["many", "few"])
def test_nonfinite_scales(dtype, seqs):
    """Rows that see such a record are not finite, the others as without it."""
    rng = np.random.default_rng(10)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 16, 2, 16, dtype)
    n0 = seqs[0][0]
    hurt = {0: 900 - n0 + 5, 1: 900 - 3}      # KV head: the first position that is hurt
    rows[1][0, 0, hurt[0]] = np.nan
    rows[3][0, 1, hurt[1]] = np.inf
    pool, tables = sv.to_pool(rng, rows, lens, 16, tables.shape[1])
    clean = [x.copy() for x in rows]
    clean[1][0, 0, hurt[0]] = clean[3][0, 1, hurt[1]] = 1.0
    want = pf.attention(q.double().numpy(), clean, starts, lens, quats, 2)
    out = attend(q, pool, tables, starts, lens, quats).cpu()
    bad = np.zeros(q.shape[:2], bool)
    for g, p in hurt.items():
        bad[p - (900 - n0):n0, 8 * g:8 * g + 8] = True
    assert not torch.isfinite(out[torch.from_numpy(bad)]).all(-1).any(), "a row that sees it is finite"
    pf.check_attention(out[torch.from_numpy(~bad)], tuple(x[~bad] for x in want), dtype, "scales")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("n", [9, 90])
def test_masked_places(dtype, n):
    """What no row sees may be anything: scales, records, page entries."""
    rng = np.random.default_rng(11)
    window, sinks, total = 100, 20, 1000
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, [(n, total)], 16, 2, 16, dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2, window, sinks)
    lo = total - n - window + 1               # the first position of the first window
    for i, x in ((1, np.nan), (3, np.inf)):
        rows[i][0, :, sinks:lo] = x
    pool, tables = sv.to_pool(rng, rows, lens, 16, tables.shape[1])
    for k in range(32 // 16 + 1, lo // 32 * 2 - 1):       # pages without a seen tile
        tables[0, k] = (-1, 1 << 30, -(1 << 31))[k % 3]
    tables[0, -(-total // 16):] = 1 << 29
    out = attend(q, pool, tables, starts, lens, quats, window=window, n_sinks=sinks)
    pf.check_attention(out, want, dtype, f"masked {n}")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_bad_pages(dtype):
    """Seen entries outside the pools: no access outside them, other sequences as they were."""
    rng = np.random.default_rng(12)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, [(50, 300), (50, 200)], 16, 2,
                                                                16, dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2)
    tables[0, 3], tables[0, 7], tables[0, 18] = -1, len(pool[0]), (1 << 31) - 1
    out = attend(q, pool, tables, starts, lens, quats)
    pf.check_attention(out[50:], tuple(x[50:] for x in want), dtype, "beside bad pages")


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_value_scales_far_apart(dtype):
    """Value scales over 2^12: the bounds hold, whose errors are in parts of the weighted scale."""
    rng = np.random.default_rng(13)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, [(70, 500)], 16, 2, 16, dtype)
    rows[3] = rows[3] * np.exp2(rng.uniform(-6, 6, rows[3].shape)).astype(np.float32)
    pool, tables = sv.to_pool(rng, rows, lens, 16, tables.shape[1])
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2)
    pf.check_attention(attend(q, pool, tables, starts, lens, quats), want, dtype, "value scales")


# ---- arguments --------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_strides_and_scale(dtype):
    rng = np.random.default_rng(14)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, [(70, 300), (2, 50)], 16, 2, 64,
                                                                dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2, scale=0.05)
    wide = torch.zeros(q.shape[0], 20, D, dtype=dtype, device=sv.DEV)
    wide[:, 2:18] = q.to(sv.DEV)
    out = torch.full((q.shape[0], 17, D), 3.0, dtype=dtype, device=sv.DEV)
    got = attend(wide[:, 2:18], pool, tables, starts, lens, quats, out=out[:, 1:], softmax_scale=0.05)
    assert got.data_ptr() == out[:, 1:].data_ptr()
    pf.check_attention(out[:, 1:], want, dtype, "strides")
    assert torch.all(out[:, 0] == 3.0)


def test_row_starts_as_they_come():
    """Values outside the tokens and descending pairs: taken as said, nothing outside written."""
    rng = np.random.default_rng(15)
    seqs = [(20, 60), (7, 30), (9, 50)]
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 16, 2, 16, torch.float16)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 2)
    given = np.array([-5, 20, 27, 10 ** 9], np.int32)         # 0, .., 36
    out = attend(q, pool, tables, given, lens, quats)
    pf.check_attention(out, want, torch.float16, "row starts")
    given = np.array([20, 0, 20, 27], np.int32)               # none, the first's tokens, 7
    out = torch.full(q.shape, 5.0, dtype=q.dtype, device=sv.DEV)
    attend(q, pool, tables, given, lens, quats, out=out)
    assert torch.all(out[27:] == 5.0) and torch.isfinite(out).all()


def test_lengths_beyond_max():
    """seq_lens above max_seq_len count as it."""
    rng = np.random.default_rng(16)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, [(30, 160), (4, 100)], 16, 2, 16,
                                                                torch.float16)
    a = attend(q, pool, tables, starts, np.array([160, 100], np.int32), quats, max_seq_len=160)
    b = attend(q, pool, tables, starts, np.array([10 ** 6, 100], np.int32), quats, max_seq_len=160)
    assert torch.equal(a, b)


# ---- many sequences ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("batch,long", [(1100, 0), (4200, 0), (1500, 400)])
def test_many_sequences(dtype, batch, long):
    """More sequences than are listed at a time, some without tokens; a long one among them."""
    rng = np.random.default_rng(batch)
    seqs = [(int(n), int(n + c)) for n, c in zip(rng.integers(0, 3, batch), rng.integers(0, 40, batch))]
    if long:
        seqs[1030] = (long, 2 * long)
    rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 2, 1, 16, dtype)
    want = pf.attention(q.double().numpy(), rows, starts, lens, quats, 1)
    out = attend(q, pool, tables, starts, lens, quats)
    pf.check_attention(out, want, dtype, f"{batch} sequences")


@pytest.mark.parametrize("rows,n_pages", [(9000, 30000), (20, 4300000), (8192, 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend_many(rows, n_pages, in_place):
    """Sequences and pages on both sides of the limits of two launches."""
    rng = np.random.default_rng([rows, n_pages])
    tables, lens, more, refs = extend_case(rng, rows, 16, 6, n_pages, 60, 30, 1, True)
    refs[refs < 0] = 1                         # (the free ones are few, far apart)
    refs[rng.random(n_pages) < 0.5] = 1
    n = int(np.maximum(more, 0).sum()) + 3
    want = pf.extend(tables, lens, more, refs, 16, n)
    t, ln, m, r = (sv.dev(x) for x in (tables, lens, more, refs))
    status = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    kw = {} if in_place else {"out_tables": torch.full_like(t, 77), "out_lens": torch.full_like(ln, 77),
                              "out_refs": torch.full_like(r, 77)}
    got = api.iq_extend_pages(t, ln, m, r, 16, n_tokens=n, status=status, **kw)
    for name, x, y in zip(("row_starts", "slots", "positions", "tables", "lens", "refs"), got, want):
        assert np.array_equal(x.cpu().numpy(), y), name
    assert int(status) == want[6]


def test_large_pool():
    """Records beyond 2^32 bytes of a pool: slots, compression and attention there."""
    hkv, page, n_pages = 4, 64, 360000
    pool = {}
    for s in "kv":
        pool[s + "_codes"] = torch.empty((n_pages, hkv, page, 48), dtype=torch.uint8, device=sv.DEV)
        pool[s + "_norms"] = torch.empty((n_pages, hkv, page), device=sv.DEV)
    assert pool["k_codes"].numel() > 1 << 32
    refs = torch.ones(n_pages, dtype=torch.int32, device=sv.DEV)
    used = 5
    refs[-used:] = 0
    tables = torch.full((1, 8), -1, dtype=torch.int32, device=sv.DEV)
    lens = torch.zeros(1, dtype=torch.int32, device=sv.DEV)
    n = used * page - 9
    more = torch.full((1,), n, dtype=torch.int32, device=sv.DEV)
    starts, slots, positions, *_ = api.iq_extend_pages(tables, lens, more, refs, page, n_tokens=n)
    assert int(slots[0]) == (n_pages - used) * page and int(slots[-1]) == (n_pages * page - 10)
    rng = np.random.default_rng(17)
    kv = torch.from_numpy(rng.standard_normal((2, n, hkv, D))).half().to(sv.DEV)
    quats = sv.dev(sv.rotation(3, hkv))
    api.iq_compress_kv_slots(kv[0], kv[1], quats, pool, slots)
    rows = [pool[x][-used:].transpose(0, 1).reshape(1, hkv, used * page, *pool[x].shape[3:]).cpu().numpy()
            for x in sv.NAMES]
    q = torch.from_numpy(rng.standard_normal((n, 2 * hkv, D))).half()
    want = pf.attention(q.double().numpy(), rows, starts.cpu().numpy(), [n], quats.cpu().numpy(), hkv)
    out = api.iq_prefill_attention_paged(q.to(sv.DEV), pool, tables, starts, lens, quats)
    pf.check_attention(out, want, torch.float16, "large pool")


# ---- a serving step's operators together --------------------------------------------------------
def tensors(seed, steps, batch, hq, hkv, page, n_pages, width, dtype, n_tokens):
    """The state of a server and every step's new lengths and projections."""
    rng = np.random.default_rng(seed)
    pool = {}
    for s in "kv":
        pool[s + "_codes"] = torch.zeros((n_pages, hkv, page, 48), dtype=torch.uint8, device=sv.DEV)
        pool[s + "_norms"] = torch.zeros((n_pages, hkv, page), device=sv.DEV)
    state = dict(pool=pool, quats=sv.dev(sv.rotation(21, hkv)),
                 freqs=api.iq_rope_frequencies(D, theta=1e5, scaling="bands", factor=4.0).to(sv.DEV),
                 tables=torch.full((batch, width), -1, dtype=torch.int32, device=sv.DEV),
                 lens=torch.zeros(batch, dtype=torch.int32, device=sv.DEV),
                 refs=torch.zeros(n_pages, dtype=torch.int32, device=sv.DEV),
                 more=torch.zeros(batch, dtype=torch.int32, device=sv.DEV),
                 starts=torch.zeros(batch + 1, dtype=torch.int32, device=sv.DEV),
                 slots=torch.zeros(n_tokens, dtype=torch.int64, device=sv.DEV),
                 positions=torch.zeros(n_tokens, dtype=torch.int32, device=sv.DEV),
                 status=torch.zeros(1, dtype=torch.int32, device=sv.DEV),
                 qkv=torch.zeros((n_tokens, hq + 2 * hkv, D), dtype=dtype, device=sv.DEV),
                 out=torch.zeros((n_tokens, hq, D), dtype=dtype, device=sv.DEV),
                 ws=torch.empty(api.iq_prefill_workspace_bytes(batch, n_tokens, hq, hkv, width * page),
                                dtype=torch.uint8, device=sv.DEV),
                 xs=torch.empty(api.iq_extend_workspace_bytes(n_pages, batch), dtype=torch.uint8,
                                device=sv.DEV))
    plan = []
    for i in range(steps):
        more = rng.integers(0, 2, batch) if i % 2 else rng.integers(0, 90, batch)
        x = torch.from_numpy(rng.standard_normal((n_tokens, hq + 2 * hkv, D))).to(dtype)
        plan.append((more.astype(np.int32), x))
    return state, plan


def serve(s, page, hq, hkv):
    """One step, everything in place, q and k slices of one projection's output."""
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
    api.iq_extend_pages(s["tables"], s["lens"], s["more"], s["refs"], page, row_starts=s["starts"],
                        slots=s["slots"], positions=s["positions"], out_tables=s["tables"],
                        out_lens=s["lens"], out_refs=s["refs"], workspace=s["xs"], status=s["status"])
    api.iq_rotate_positions(q, k, s["positions"], s["freqs"], q_out=q, k_out=k)
    api.iq_compress_kv_slots(k, v, s["quats"], s["pool"], s["slots"])
    api.iq_prefill_attention_paged(q, s["pool"], s["tables"], s["starts"], s["lens"], s["quats"],
                                   out=s["out"], workspace=s["ws"])


def rows_of(s, page):
    """The records of every sequence, [B][H][cap][..], from the pools."""
    tables = s["tables"].cpu().numpy()
    at = np.where(tables >= 0, tables, 0)
    out = []
    for x in sv.NAMES:
        a = s["pool"][x].cpu().numpy()[at]               # [B][pages][H][page][..]
        a = np.moveaxis(a, 2, 1)
        out.append(a.reshape(a.shape[0], a.shape[1], -1, *a.shape[4:]))
    return out


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("batch,hq,hkv,page", [(5, 16, 2, 16), (3, 4, 4, 64)])
def test_serving_steps(dtype, batch, hq, hkv, page):
    """Several steps of chunks and single tokens: pages and slots by the plain form, rotated queries
    and keys in 64 bits, records those of the bulk compression, outputs in 64 bits over them; at the
    end a decode step over the same pools."""
    n_pages, width, n_tokens = 500 // page * batch, 400 // page, 90 * batch
    s, plan = tensors(33, 4, batch, hq, hkv, page, n_pages, width, dtype, n_tokens)
    for more, x in plan:
        before = [s[n].cpu().numpy().copy() for n in ("tables", "lens", "refs")]
        want = pf.extend(before[0], before[1], more, before[2], page, n_tokens)
        s["more"].copy_(torch.from_numpy(more))
        s["qkv"].copy_(x)
        s["out"].fill_(4.0)
        serve(s, page, hq, hkv)
        for name, y in zip(("starts", "slots", "positions", "tables", "lens", "refs"), want):
            assert np.array_equal(s[name].cpu().numpy(), y), name
        assert int(s["status"]) == 0
        n = int(more.sum())
        rot = s["qkv"].cpu()
        ref = pf.rope(x[:, :hq + hkv].double().numpy(), want[2], s["freqs"].cpu().numpy(), "half")
        # (tests of the rotation alone derive this: 2^-21.3 and half a step of the type, of 6.5)
        tol = 6.5 * (2.0 ** -21 + (2.0 ** -11 if dtype == torch.float16 else 2.0 ** -24))
        assert np.abs(rot[:, :hq + hkv].double().numpy() - ref).max() <= tol
        if n == 0:
            continue
        # the records of the new tokens
        cache = api.alloc_cache(1, hkv, -(-n // 16) * 16, sv.DEV)
        kv = s["qkv"][:n, hq:].transpose(0, 1)
        api.iq_compress_kv(kv[:hkv].contiguous()[None], kv[hkv:].contiguous()[None], s["quats"],
                           cache["k_codes"], cache["k_norms"], cache["v_codes"], cache["v_norms"])
        at = s["slots"][:n]
        for name in sv.NAMES:
            got = s["pool"][name][at // page, :, at % page]
            src = cache[name][0].transpose(0, 1)[:n]
            if got.dtype == torch.uint8:
                # (a coordinate at the border of two codes may get either)
                assert (got != src).float().mean() <= 1e-4, name
            else:
                assert ((got - src).abs() <= 2.0 ** -22 * src).all(), name
        starts, lens = want[0], want[4]
        ref = pf.attention(rot[:, :hq].double().numpy(), rows_of(s, page), starts, lens,
                           s["quats"].cpu().numpy(), hkv)
        pf.check_attention(s["out"][:n], tuple(a[:n] for a in ref), dtype, f"step of {n}")
        assert torch.all(s["out"][n:] == 4.0), "padding was written"
    # the last token of each sequence, by the decode kernel
    last = (s["starts"][1:] - 1).long()
    some = (s["starts"][1:] > s["starts"][:-1]).cpu()
    dec = api.iq_decode_attention_paged(s["qkv"][last][:, :hq].float().contiguous(), s["pool"],
                                        s["tables"], s["lens"], s["quats"])
    err = (dec - s["out"][last].float()).cpu()[some]
    # (of one row: its bound of the 64-bit test with B <= 40, |v| <= 30; fp32: both within 4e-6)
    lim = (2.0 ** -11 * 82 * 30 if dtype == torch.float16 else 1e-4)
    assert some.any() and err.norm(dim=-1).max() <= lim


def test_serving_graph():
    """A step as one graph, replayed for other lengths and values, with eager work between: as
    the eager step on a state of its own, bit for bit; two graphs on two streams beside each other."""
    batch, hq, hkv, page, width, n_tokens = 4, 16, 2, 16, 40, 420
    a, plan = tensors(34, 6, batch, hq, hkv, page, 300, width, torch.float16, n_tokens)
    b, _ = tensors(34, 6, batch, hq, hkv, page, 300, width, torch.float16, n_tokens)
    c, _ = tensors(34, 6, batch, hq, hkv, page, 300, width, torch.float16, n_tokens)
    graphs = []
    for s in (a, c):
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            serve(s, page, hq, hkv)               # (no new tokens: nothing changes)
        torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            serve(s, page, hq, hkv)
        graphs.append((g, torch.cuda.Stream()))
    for more, x in plan:
        for s in (a, b, c):
            s["more"].copy_(torch.from_numpy(more))
            s["qkv"].copy_(x)
            s["out"].zero_()
        torch.cuda.synchronize()
        for g, stream in graphs:
            with torch.cuda.stream(stream):
                g.replay()
        serve(b, page, hq, hkv)
        torch.cuda.synchronize()
        for s in (a, c):
            for name in ("tables", "lens", "refs", "starts", "slots", "positions", "status", "qkv",
                         "out"):
                assert torch.equal(s[name], b[name]), name
            for name in sv.NAMES:
                assert torch.equal(s["pool"][name], b["pool"][name]), name
        float((b["out"].float() ** 2).sum())      # eager work between the replays
    assert int(b["lens"].sum()) > 100


def test_two_streams():
    """Two calls at once, each with a workspace of its own, on streams other than the current one."""
    rng = np.random.default_rng(18)
    cases, outs = [], []
    for seqs in ([(200, 800)], MIXED):
        rows, lens, starts, pool, tables, quats, q = attention_case(rng, seqs, 16, 2, 16, torch.float16)
        cases.append([q.to(sv.DEV), sv.as_dict(pool)] + [sv.dev(x) for x in (tables, starts, lens, quats)])
    alone = [api.iq_prefill_attention_paged(*c) for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for c in cases:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                got.append(api.iq_prefill_attention_paged(*c))
        torch.cuda.synchronize()
        for x, y in zip(got, alone):
            assert torch.equal(x, y)


# ---- the binding --------------------------------------------------------------------------------
class General:   # a native module that never calls
    def __getattr__(self, name):
        return lambda *a: None


def test_both_paths_agree(monkeypatch):
    """The native checks and the general path: the same results, with outputs given and made."""
    got = []
    for general in (False, True):
        if general:
            monkeypatch.setattr(_lib, "native", lambda: General())
        s, plan = tensors(35, 3, 3, 16, 2, 16, 120, 30, torch.float16, 260)
        for more, x in plan:
            s["more"].copy_(torch.from_numpy(more))
            s["qkv"].copy_(x)
            serve(s, 16, 16, 2)
        new = [api.iq_extend_pages(s["tables"].clone(), s["lens"].clone(), s["more"], s["refs"].clone(),
                                   16, n_tokens=260),
               api.iq_rotate_positions(s["qkv"][:, :16], s["qkv"][:, 16:18], s["positions"], s["freqs"],
                                       layout="interleaved", amplitude=0.5),
               (api.iq_prefill_attention_paged(s["qkv"][:, :16], s["pool"], s["tables"], s["starts"],
                                               s["lens"], s["quats"], window=9, n_sinks=2),)]
        got.append([s[n].clone() for n in ("tables", "lens", "refs", "starts", "slots", "positions",
                                           "status", "qkv", "out")]
                   + [s["pool"][n].clone() for n in sv.NAMES] + [y.clone() for t in new for y in t])
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("general", [False, True])
@pytest.mark.parametrize("wrong,error", [
    ({"q": lambda t: t.bfloat16()}, TypeError), ({"q": lambda t: t[:, :, :64]}, ValueError),
    ({"q": lambda t: t.cpu()}, ValueError), ({"q": lambda t: t.transpose(0, 1)}, ValueError),
    ({"out": lambda t: t.float()}, TypeError), ({"out": lambda t: t[:-1]}, ValueError),
    ({"out": "q"}, _lib.IsoQuantError), ({"ws": lambda t: t[:256]}, _lib.IsoQuantError),
    ({"lens": lambda t: t.long()}, TypeError), ({"lens": lambda t: t[:-1]}, ValueError),
    ({"starts": lambda t: t[:-1]}, ValueError), ({"tables": lambda t: t[:, ::2]}, ValueError),
    ({"quats": lambda t: t[:1]}, ValueError), ({"most": lambda m: 10 ** 6}, _lib.IsoQuantError),
    ({"window": lambda m: -1}, _lib.IsoQuantError)])
def test_wrong_attention_arguments(monkeypatch, general, wrong, error):
    if general:
        monkeypatch.setattr(_lib, "native", lambda: General())
    s, _ = tensors(36, 0, 3, 16, 2, 16, 120, 30, torch.float16, 60)
    a = dict(q=s["qkv"][:, :16], out=s["out"], ws=s["ws"], lens=s["lens"], starts=s["starts"],
             tables=s["tables"], quats=s["quats"], most=None, window=0)
    for name, f in wrong.items():
        a[name] = a[f] if isinstance(f, str) else f(a[name])
    with pytest.raises(error):
        api.iq_prefill_attention_paged(a["q"], s["pool"], a["tables"], a["starts"], a["lens"], a["quats"],
                                       window=a["window"], out=a["out"], workspace=a["ws"],
                                       max_seq_len=a["most"])


@pytest.mark.parametrize("general", [False, True])
def test_wrong_other_arguments(monkeypatch, general):
    if general:
        monkeypatch.setattr(_lib, "native", lambda: General())
    s, _ = tensors(37, 0, 3, 16, 2, 16, 120, 30, torch.float16, 60)
    q, k, v = s["qkv"][:, :16], s["qkv"][:, 16:18], s["qkv"][:, 18:]
    for error, call in (
            (TypeError, lambda: api.iq_rotate_positions(q, k, s["positions"].long(), s["freqs"])),
            (TypeError, lambda: api.iq_rotate_positions(q, k.float(), s["positions"], s["freqs"])),
            (TypeError, lambda: api.iq_rotate_positions(q, k, s["positions"], s["freqs"].float())),
            (ValueError, lambda: api.iq_rotate_positions(q, k[:-1], s["positions"], s["freqs"])),
            (_lib.IsoQuantError, lambda: api.iq_rotate_positions(q, k, s["positions"], s["freqs"][:12])),
            (_lib.IsoQuantError, lambda: api.iq_rotate_positions(q, k, s["positions"], s["freqs"],
                                                                 k_out=q[:, :2])),
            (TypeError, lambda: api.iq_compress_kv_slots(k, v, s["quats"], s["pool"], s["slots"].int())),
            (ValueError, lambda: api.iq_compress_kv_slots(k, v, s["quats"], s["pool"], s["slots"][1:])),
            (ValueError, lambda: api.iq_compress_kv_slots(q, None, s["quats"], s["pool"], s["slots"])),
            (TypeError, lambda: api.iq_extend_pages(s["tables"], s["lens"].long(), s["more"], s["refs"], 16,
                                                    n_tokens=60)),
            (ValueError, lambda: api.iq_extend_pages(s["tables"], s["lens"], s["more"][1:], s["refs"], 16,
                                                     n_tokens=60)),
            (_lib.IsoQuantError, lambda: api.iq_extend_pages(s["tables"], s["lens"], s["more"], s["refs"],
                                                             24, n_tokens=60)),
            (_lib.IsoQuantError, lambda: api.iq_extend_pages(s["tables"], s["lens"], s["more"], s["refs"],
                                                             16, n_tokens=60, out_lens=s["more"]))):
        with pytest.raises(error):
            call()


def test_no_tokens():
    """Steps without tokens, arrays of none: nothing happens, nothing fails."""
    s, _ = tensors(38, 0, 3, 16, 2, 16, 120, 30, torch.float16, 8)
    none = {n: s[n][:0] for n in ("qkv", "slots", "positions", "out")}
    starts, slots, positions, *_ = api.iq_extend_pages(s["tables"], s["lens"], s["more"], s["refs"], 16,
                                                       n_tokens=0, status=s["status"])
    assert not starts.any() and slots.numel() == positions.numel() == 0 and int(s["status"]) == 0
    q, k = api.iq_rotate_positions(none["qkv"][:, :16], none["qkv"][:, 16:18], none["positions"], s["freqs"])
    assert q.shape == (0, 16, D) and k.shape == (0, 2, D)
    before = s["pool"]["k_codes"].clone()
    api.iq_compress_kv_slots(k, k, s["quats"], s["pool"], none["slots"])
    assert torch.equal(before, s["pool"]["k_codes"])
    out = api.iq_prefill_attention_paged(q, s["pool"], s["tables"], starts, s["lens"], s["quats"])
    assert out.shape == (0, 16, D)
    # tokens that are all padding
    out = torch.full((8, 16, D), 2.0, dtype=torch.float16, device=sv.DEV)
    api.iq_prefill_attention_paged(s["qkv"][:, :16], s["pool"], s["tables"], s["starts"], s["lens"],
                                   s["quats"], out=out)
    assert torch.all(out == 2.0)
