"""The operators of a speculative step against their oracle in 64 bits, through the binding."""
import numpy as np
import pytest
import torch

from oracle import step as O
from paper_2604_07609_b200 import binding as B
from synth import model_cfg

pytestmark = pytest.mark.gpu

BS = 16
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}     # half a step, relative to the value
U = 2.0 ** -24


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def f64(t):
    return t.double().cpu().numpy()


def shape(rep=4, hkv=2, hd=128, dtype="bf16", layers=2):
    return model_cfg(1, n_layers=layers, n_q_heads=rep * hkv, n_kv_heads=hkv, head_dim=hd, dtype=dtype)


def new_pool(m, blocks, fill=float("nan")):
    return torch.full((m.n_layers, 2, blocks, m.n_kv_heads, BS, m.head_dim), fill, dtype=DT[m.dtype], device="cuda")


# ---- tables -----------------------------------------------------------------------------------------------------------
def tables_case(rng, n, ctx_hi, new_hi, spare, zero=0.2):
    ctx, new = rng.integers(0, ctx_hi + 1, n), rng.integers(0, new_hi + 1, n)
    new[rng.random(n) < zero] = 0
    held = np.array([-(-c // BS) + int(rng.integers(0, 3)) for c in ctx])
    stride = int(max(max(held), (-(-(ctx + new) // BS)).max())) + int(rng.integers(0, 3))
    ids = rng.permutation(int(held.sum()) + int((ctx + new).sum()) // BS + n + 5)
    table, at = np.full((n, max(stride, 1)), -1), 0
    for r in range(n):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    return ctx, new, held, ids[at:], len(ids) - at, table, int(new.sum()) + spare


def check_tables(ctx, new, held, free, count, table, rows, out=None, cap=None):
    want = O.build_tables(list(map(int, ctx)), list(map(int, new)), list(map(int, held)), free, count, table, rows)
    dev = ints(table)
    t = B.blink_build_tables(ints(ctx), ints(new), ints(held), ints(free), ints([count]), dev, max_rows=rows) if out is None else out(dev)
    got = [x.cpu().numpy() for x in t]
    for name, w, g in zip(("row_start", "kv_len", "positions", "slots", "held", "count", "status"), want, got):
        assert np.array_equal(np.atleast_1d(w), g), name
    assert np.array_equal(dev.cpu().numpy(), want[7])


@pytest.mark.parametrize("n,ctx,new,spare", [(1, 0, 1, 0), (1, 40, 1, 3), (3, 20, 40, 5), (31, 100, 3, 0), (256, 300, 8, 77), (257, 60, 33, 1),
                                             (1025, 50, 2, 0), (4096, 30, 3, 9), (40, 2000, 700, 100), (200, 50, 600, 9),
                                             (3, 0, 20000, 70000)])
def test_tables(n, ctx, new, spare):
    case = list(tables_case(np.random.default_rng(n), n, ctx, new, spare))
    case[6] = max(1, case[6])
    check_tables(*case)


def test_tables_hand_out_nothing_when_refused():
    rng = np.random.default_rng(5)
    ctx, new, held, free, count, table, rows = tables_case(rng, 40, 50, 40, 3, zero=0)
    need = int(np.maximum(0, -(-(ctx + new) // BS) - held).sum())
    check_tables(ctx, new, held, free, need, table, rows)            # exactly enough
    check_tables(ctx, new, held, free, need - 1, table, rows)
    check_tables(ctx, new, held, free, len(free) + 1, table, rows)
    check_tables(ctx, new, held, free, -1, table, rows)
    check_tables(ctx, new, held, free, count, table, int(new.sum()) - 1)
    check_tables(ctx, new, held, free, count, table[:, :-(-int((ctx + new).max()) // BS) - 1], rows) if (held < table.shape[1] - 1).all() else None
    for a in (ctx, new, held):
        b = a.copy()
        b[17] = -1
        args = [b if x is a else x for x in (ctx, new, held)]
        check_tables(*args, free, count, table, rows)


def test_tables_in_place_and_entries_that_are_no_block():
    rng = np.random.default_rng(6)
    ctx, new, held, free, count, table, rows = tables_case(rng, 300, 90, 20, 40)
    table[5, 0], table[9, 0] = -1, 1 << 28
    ctx[5] = ctx[9] = 0
    held[5] = held[9] = 1

    def run(dev):
        h, c = ints(held), ints([count])
        out = B.make_step_tables(len(ctx), rows, "cuda")._replace(blocks_held=h, free_count=c)
        return B.blink_build_tables(ints(ctx), ints(new), h, ints(free), c, dev, out=out)
    check_tables(ctx, new, held, free, count, table, rows, run)


# ---- norms, rotation, cache -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [1, 3, 64, 300, 3001])   # (the last: several groups of heads a warp)
@pytest.mark.parametrize("rep,hkv,hd,dtype,qkv", [(4, 2, 128, "bf16", "bf16"), (1, 3, 64, "bf16", "bf16"), (8, 1, 128, "bf16", "fp32"), (2, 2, 64, "fp32", "fp32"),
                                                  (4, 8, 64, "bf16", "fp32"), (1, 1, 128, "fp32", "fp32")])
@pytest.mark.parametrize("gains", ["both", "q", None])
def test_norm_rope(rows, rep, hkv, hd, dtype, qkv, gains):
    m = shape(rep, hkv, hd, dtype, layers=3).with_(rope_theta=5e5)
    rng = np.random.default_rng(rows * 7 + hd)
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, m.qkv_dim + 8, device="cuda", generator=g).mul_(2).to(DT[qkv])[:, :m.qkv_dim]     # rows further apart
    qg = 1 + 0.3 * torch.randn(hd, device="cuda", generator=g) if gains else None
    kg = 1 + 0.3 * torch.randn(hd, device="cuda", generator=g) if gains == "both" else None
    pos = rng.integers(0, 1 << 30, rows) if rows == 64 else rng.integers(0, 6000, rows)
    blocks = rows // BS + 4
    slots = rng.permutation(blocks * BS)[:rows]
    pool = new_pool(m, blocks, 3.0)
    out = torch.full((rows, m.q_dim + 16), 5.0, dtype=DT[dtype], device="cuda")
    if rows > 2:
        pos[1] = -1                              # left alone
        slots[2] = -1 if rows < 100 else blocks * BS
    B.blink_qk_norm_rope(m, pool, 1, x, qg, kg, ints(pos), ints(slots), out=out[:, :m.q_dim])
    xs = f64(x).reshape(rows, m.n_q_heads + 2 * hkv, hd)
    Hq = m.n_q_heads
    # sums of hd squares in runs of 16 and a tree (20 roundings, halved by the root), rsqrtf 2 ulp, three products, angles to 2 ulp of
    # one and two products and a sum of the rotation: 24 roundings of the terms' size at most
    for heads, gain, got in ((slice(0, Hq), qg, f64(out[:, :m.q_dim]).reshape(rows, Hq, hd)),
                             (slice(Hq, Hq + hkv), kg, None), (slice(Hq + hkv, None), "v", None)):
        y, size = (xs[:, heads], 0 * xs[:, heads]) if isinstance(gain, str) else O.norm_rope(xs[:, heads], None if gain is None else f64(gain), np.maximum(pos, 0), 5e5, m.rms_eps)
        tol = HALF[dtype] * abs(y) + 24 * U * size
        if got is not None:
            live = pos >= 0
            assert (abs(got - y)[live] <= tol[live]).all()
            assert (got[~live] == 5.0).all()
        else:
            kv = f64(pool[1, 1 if isinstance(gain, str) else 0]).transpose(0, 2, 1, 3).reshape(blocks * BS, hkv, hd)
            live = (pos >= 0) & (slots >= 0) & (slots < blocks * BS)
            assert (abs(kv[slots[live]] - y[live]) <= tol[live]).all()
            kv[slots[live]] = 3.0
            assert (kv == 3.0).all()             # nothing else was written
    assert (out[:, m.q_dim:] == 5.0).all() and (pool[0] == 3.0).all() and (pool[2] == 3.0).all()


def test_norm_rope_in_place_and_special_rows():
    m = shape(2, 2, 64)
    x = torch.randn(40, m.qkv_dim, device="cuda").bfloat16()
    x[3] = 0                                     # a head of zeros stays one: eps
    x[5, 70] = float("inf")
    pos, slots = ints(np.arange(40)), ints(np.arange(40))
    want = B.blink_qk_norm_rope(m, new_pool(m, 3, 0.0), 0, x.clone(), torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), pos, slots)
    assert (want[3] == 0).all() and torch.isnan(want[5, 64:128]).any() and not torch.isnan(want[5, :64]).any()
    y = x.clone()
    B.blink_qk_norm_rope(m, new_pool(m, 3, 0.0), 0, y, torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), pos, slots, out=y[:, :m.q_dim])
    assert torch.equal(y[:, :m.q_dim].nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(y[:, m.q_dim:], x[:, m.q_dim:])


# ---- attention --------------------------------------------------------------------------------------------------------
def attention_case(m, ctx, new, window, sinks, seed=0, pad=0, layer=1, q_pad=0, scale=1.0):
    """Inputs of requests with ctx cached tokens and new rows; everything that no row of its request sees is NaN, and blocks that hold
    nothing else have no entry in the table."""
    rng = np.random.default_rng(seed)
    ctx, new = np.asarray(ctx), np.asarray(new)
    n, hd, hkv = len(ctx), m.head_dim, m.n_kv_heads
    start = np.concatenate([[0], np.cumsum(new)])
    rows = int(start[-1]) + pad
    seen = [sorted(set().union(*[O.visible(c + i, window, sinks) for i in range(k)]) if k else []) for c, k in zip(ctx, new)]
    used = [sorted({j // BS for j in s}) for s in seen]
    total = sum(map(len, used)) + 3
    ids = rng.permutation(total)
    table = np.where(rng.random((n, int(max(1, (-(-(ctx + new) // BS)).max())) + 1)) < 0.5, -1, 1 << 30)
    pool = new_pool(m, total)
    g = torch.Generator(device="cuda").manual_seed(seed)
    at, kv = 0, []
    for r in range(n):
        table[r, used[r]] = ids[at:at + len(used[r])]
        at += len(used[r])
        k, v = (torch.randn(len(seen[r]), hkv, hd, device="cuda", generator=g).to(pool.dtype) for _ in (0, 1))
        if seen[r]:
            j = np.array(seen[r])
            block = torch.from_numpy(table[r, j // BS]).cuda()
            pool[layer, 0][block, :, torch.from_numpy(j % BS).cuda()] = k
            pool[layer, 1][block, :, torch.from_numpy(j % BS).cuda()] = v
        full = np.full((2, int(ctx[r] + new[r]), hkv, hd), np.nan)
        if seen[r]:
            full[0, j], full[1, j] = f64(k), f64(v)
        kv.append(full)
    q = (scale * torch.randn(max(1, rows), m.q_dim + q_pad, device="cuda", generator=g)).to(pool.dtype)[:, :m.q_dim]
    return dict(m=m, pool=pool, layer=layer, q=q, row_start=ints(start), kv_len=ints(ctx + new), table=ints(table), window=window, sinks=sinks, start=start, ctx=ctx, kv=kv)


def run_attention(c, max_new=None, **kw):
    longest = max(1, int(np.diff(c["start"]).max()))
    return B.blink_window_attention(c["m"], c["pool"], c["layer"], c["q"], c["row_start"], c["kv_len"], c["table"], c["window"], c["sinks"],
                                    longest if max_new is None else max_new, **kw)


def check_attention(c, out, only=None):
    """Bound of the error: half a step of the output; in bf16 half a step of each probability in its product with the values (their sum
    is taken before that rounding); scores to (hd + 8) roundings of their products' sum, which enter a probability as they are; 2^-20
    for the exponentials, and a rounding per key of the running sums."""
    m, start = c["m"], c["start"]
    q, got = f64(c["q"]), f64(out)
    for r in range(len(c["ctx"])) if only is None else only:
        a, b = start[r], start[r + 1]
        if a == b:
            continue
        keys, values = c["kv"][r]
        want, size, spread = O.window_attention(q[a:b].reshape(b - a, m.n_q_heads, m.head_dim), keys, values, c["ctx"][r], c["window"], c["sinks"])
        p = 2.0 ** -8 if m.dtype == "bf16" else 0.0
        tol = HALF[m.dtype] * abs(want) + size * (p * 1.01 + 2 * (m.head_dim + 8) * U * spread[..., None] + 2.0 ** -20 + len(keys) * U)
        err = abs(got[a:b].reshape(want.shape) - want)
        assert (err <= tol).all(), f"request {r}: {np.nanmax(err / np.maximum(tol, 1e-30)):.2f} of the bound, {np.isnan(err).sum()} NaN"


SHAPES = [(4, 2, 128, "bf16"), (1, 2, 128, "bf16"), (8, 1, 64, "bf16"), (2, 3, 64, "bf16"), (4, 1, 64, "fp32"), (8, 1, 128, "fp32"), (1, 2, 128, "fp32")]


@pytest.mark.parametrize("rep,hkv,hd,dtype", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (16, 4), (17, 1), (50, 20), (1000, 4), (33, 64)])
def test_attention_single_rows(rep, hkv, hd, dtype, window, sinks):
    c = attention_case(shape(rep, hkv, hd, dtype), [0, 1, 14, 15, 16, 31, 47, 63, 200, 333], [1] * 10, window, sinks, seed=window)
    check_attention(c, run_attention(c))


@pytest.mark.parametrize("rep,hkv,hd,dtype", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 2), (20, 4), (64, 0), (150, 33)])
def test_attention_drafts(rep, hkv, hd, dtype, window, sinks):
    c = attention_case(shape(rep, hkv, hd, dtype), [0, 15, 100, 7, 260, 64, 30], [3, 4, 1, 0, 2, 5, 8], window, sinks, seed=window, pad=2, q_pad=8)
    out = torch.full((c["q"].shape[0], c["m"].q_dim + 8), 9.0, dtype=c["q"].dtype, device="cuda")
    run_attention(c, out=out[:, :c["m"].q_dim])
    check_attention(c, out[:, :c["m"].q_dim])
    assert (out[-2:] == 9.0).all() and (out[:, c["m"].q_dim:] == 9.0).all()


@pytest.mark.parametrize("rep,hkv,hd,dtype", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 4), (130, 0), (1, 1), (0, 7)])
def test_attention_prompts(rep, hkv, hd, dtype, window, sinks):
    c = attention_case(shape(rep, hkv, hd, dtype), [0, 33, 0, 5, 200], [65, 40, 129, 1, 100], window, sinks, seed=window, pad=3)
    out = torch.full((c["q"].shape[0], c["m"].q_dim), 9.0, dtype=c["q"].dtype, device="cuda")
    run_attention(c, out=out)
    check_attention(c, out)
    assert (out[-3:] == 9.0).all()


@pytest.mark.parametrize("rep,hkv,hd,dtype", [(4, 1, 128, "bf16"), (8, 2, 64, "bf16"), (4, 1, 64, "fp32"), (1, 1, 128, "fp32")])
def test_attention_a_long_context_is_shared_out_and_joined(rep, hkv, hd, dtype):
    for window, sinks in ((0, 0), (4000, 5)):
        c = attention_case(shape(rep, hkv, hd, dtype), [6001, 3, 2500], [1, 1, 2], window, sinks, seed=3)
        check_attention(c, run_attention(c))


@pytest.mark.parametrize("rep,hkv,hd,dtype", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (513, 20), (700, 4), (600, 64)])
def test_attention_wide_tables(rep, hkv, hd, dtype, window, sinks):
    """Tables with room for long contexts, of which requests use little, or as much as a window: pieces of units, joined."""
    for new in ([1] * 9, [3, 1, 0, 2, 4, 1, 2, 1, 2]):
        c = attention_case(shape(rep, hkv, hd, dtype), [0, 1400, 15, 16, 800, 47, 1203, 200, 333], new, window, sinks, seed=window + len(set(new)))
        c["table"] = torch.nn.functional.pad(c["table"], (0, 1200), value=-1)
        out = run_attention(c)
        check_attention(c, out)
        assert torch.equal(out, run_attention(c))


@pytest.mark.parametrize("rep,hkv,hd,dtype,new", [(4, 2, 128, "bf16", 1), (4, 1, 128, "bf16", 6), (8, 1, 64, "bf16", 3), (1, 4, 64, "bf16", 1), (4, 1, 128, "fp32", 1)])
def test_attention_one_request_from_short_to_very_long(rep, hkv, hd, dtype, new):
    """A cluster for each unit, or pieces that are joined by small CTAs or large ones."""
    for ctx in (0, 255, 4093, 8190, 16380, 20000):
        c = attention_case(shape(rep, hkv, hd, dtype, layers=2), [ctx], [new], 0, 0, seed=ctx)
        out = run_attention(c)
        check_attention(c, out)
        assert torch.equal(out, run_attention(c))


def test_attention_rows_that_see_nothing_are_zeros():
    """More rows than cached tokens: positions below zero."""
    for dtype in ("bf16", "fp32"):
        for new in (3, 40):
            c = attention_case(shape(4, 2, 64, dtype), [0, 20], [new, 2], 8, 2, seed=1)
            kv_len = c["kv_len"].clone()
            kv_len[0] = 1                                      # the last of its rows alone is at position 0
            out = B.blink_window_attention(c["m"], c["pool"], 1, c["q"], c["row_start"], kv_len, c["table"], 8, 2, new)
            assert (out[:new - 1] == 0).all()
            check_attention(c, out, only=[1])
            kv_len[0] = 0
            assert (B.blink_window_attention(c["m"], c["pool"], 1, c["q"], c["row_start"], kv_len, c["table"], 8, 2, new)[:new] == 0).all()


def test_attention_blocks_that_are_none_are_zeros():
    """A seen entry that is no block of the pool: keys and values of zeros, wherever the rows go."""
    for new in (1, 3, 70):
        c = attention_case(shape(4, 2, 128), [100, 50], [new, 1], 0, 0, seed=2)
        for bad in (-1, c["pool"].shape[2], 1 << 30, -(1 << 31)):
            table = c["table"].clone()
            table[0, 2] = bad
            out = B.blink_window_attention(c["m"], c["pool"], 1, c["q"], c["row_start"], c["kv_len"], table, 0, 0, new)
            d = dict(c, kv=[c["kv"][0].copy(), c["kv"][1]])
            d["kv"][0][:, 32:48] = 0
            check_attention(d, out)


def test_attention_large_scores_and_out_over_q():
    c = attention_case(shape(4, 2, 128), [700, 20, 3], [1, 4, 60], 0, 0, seed=4, scale=12.0)
    out = run_attention(c)
    check_attention(c, out)
    q = c["q"].contiguous().clone()
    assert B.blink_window_attention(c["m"], c["pool"], 1, q, c["row_start"], c["kv_len"], c["table"], 0, 0, 60, out=q) is q
    assert torch.equal(q, out)


def test_attention_tiles_of_long_requests():
    """More tiles than the rings of shared memory hold, windows that cut tiles anywhere, sinks inside and outside of them."""
    for rep, hkv, hd in ((4, 1, 128), (1, 1, 128), (8, 1, 64), (2, 1, 64)):
        for window, sinks in ((0, 0), (200, 5), (511, 0), (64, 150), (700, 16)):
            c = attention_case(shape(rep, hkv, hd), [900, 0, 77], [50, 130, 1], window, sinks, seed=window + rep)
            check_attention(c, run_attention(c))


@pytest.mark.parametrize("rep,hkv,hd", [(4, 2, 128), (1, 3, 128), (8, 1, 64), (2, 2, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 3), (140, 40)])
def test_attention_few_rows_behind_many_keys(rep, hkv, hd, window, sinks):
    """Units that fill one stream of rows only, with any number of tiles, beside full ones."""
    c = attention_case(shape(rep, hkv, hd), [1500, 40, 250, 700, 3, 130, 120, 500], [17, 140, 33, 40, 260, 9, 33, 64], window, sinks, seed=rep)
    out = run_attention(c)
    check_attention(c, out)
    assert torch.equal(out, run_attention(c))


@pytest.mark.parametrize("rep,hkv,hd", [(4, 1, 128), (4, 4, 128), (8, 2, 64), (1, 8, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1600, 5)])
def test_attention_single_rows_drafts_and_prompts_in_one_call(rep, hkv, hd, window, sinks):
    """Long enough contexts that few rows and many have kernels of their own, which share a workspace."""
    c = attention_case(shape(rep, hkv, hd), [2000, 100, 1700, 0, 5], [1, 70, 4, 33, 0], window, sinks, seed=rep)
    out = run_attention(c)
    check_attention(c, out)
    assert all(torch.equal(out, run_attention(c)) for _ in range(3))


@pytest.mark.parametrize("n,window,top", [(30, 0, 700), (12, 0, 400), (30, 200, 9000), (9, 3000, 5000)])
def test_attention_batches_of_drafts(n, window, top):
    """Calls that go to the tiles whole, to the kernels for few rows, or to both, by requests, rows and keys."""
    rng = np.random.default_rng(n + window)
    for most, rep in ((2, 4), (3, 4), (6, 4), (9, 4), (2, 8)):
        new = rng.integers(0, most + 1, n)
        new[0] = most
        ctx = np.minimum(np.exp(rng.uniform(0, np.log(top), n)).astype(int), top)
        ctx[1] = top
        c = attention_case(shape(rep, 8, 64), ctx, new, window, 3 if window else 0, seed=most)
        out = run_attention(c)
        check_attention(c, out)
        assert torch.equal(out, run_attention(c))


@pytest.mark.parametrize("window,sinks", [(0, 0), (500, 20)])
def test_attention_units_of_one_stream_and_of_two(window, sinks):
    """Around the numbers of units at which their size changes, with requests in their own order and put in order."""
    m = shape(8, 8, 64)
    for n, rows in ((1, 16), (1, 17), (1, 300), (2, 290), (2, 300), (3, 310), (300, 17), (300, 1)):
        new = np.full(n, rows)
        new[n // 2:] = np.maximum(1, new[n // 2:] // 2)
        c = attention_case(m, np.arange(n) * 37 % 200 + (900 if n == 1 else 0), new, window, sinks, seed=n)
        out = run_attention(c, max_new=max(rows, 5))
        check_attention(c, out, only=range(0, n, max(1, n // 3)))
        assert torch.equal(out, run_attention(c, max_new=max(rows, 5)))


def test_attention_many_units_per_cta():
    """More units than a CTA has records for, in every CTA."""
    c = attention_case(shape(8, 8, 64), [3] * 45, [140] * 45, 40, 3, seed=7)
    out = run_attention(c)
    check_attention(c, out, only=[0, 22, 44])
    assert torch.equal(out, run_attention(c))          # who takes which unit changes nothing


@pytest.mark.parametrize("rep,hkv,hd,dtype", [(4, 1, 128, "bf16"), (4, 1, 64, "bf16"), (2, 1, 64, "fp32")])
@pytest.mark.parametrize("rising", [True, False])
def test_attention_scores_that_rise_and_fall(rep, hkv, hd, dtype, rising):
    """The largest score grows by far more than 2^8 from tile to tile, or is the first key's: every way to rescale."""
    for new in (1, 5, 90):
        c = attention_case(shape(rep, hkv, hd, dtype), [600], [new], 0, 0, seed=new)
        n = 600 + new
        d = torch.randn(hd, device="cuda")
        j = torch.arange(n, device="cuda", dtype=torch.float32)
        size = (j if rising else n - j) * (150.0 / n)
        k = (size[:, None] * d / d.norm() + 0.1 * torch.randn(n, hd, device="cuda")).to(c["pool"].dtype)
        block = c["table"][0].long()[torch.arange(n, device="cuda") // BS]
        c["pool"][1, 0][block, 0, torch.arange(n, device="cuda") % BS] = k
        c["kv"][0][0, :, 0] = f64(k)
        c["q"].copy_((d / d.norm() * 30.0).to(c["q"].dtype).repeat(rep)[None, :])
        check_attention(c, run_attention(c))


def test_attention_two_calls_at_once():
    cases = [attention_case(shape(4, 2, 128), [500, 20, 300], [1, 60, 4], 100, 4, seed=1), attention_case(shape(4, 2, 64), [90, 700], [200, 1], 0, 0, seed=2)]
    want = [run_attention(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(10):
        for i, (st, c) in enumerate(zip(streams, cases)):
            with torch.cuda.stream(st):
                got[i].append(run_attention(c))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w, x) for x in g)


def test_attention_the_workspace_says_that_no_wait_ran_out():
    c = attention_case(shape(4, 2, 128), [50, 3], [90, 1], 0, 0)
    ws = torch.full((B.blink_window_attention_workspace(c["m"], 90),), 255, dtype=torch.uint8, device="cuda")
    check_attention(c, run_attention(c, workspace=ws))
    assert int(ws[:4].view(torch.int32)) == B.BLINK_OK


def test_attention_calls_behind_one_another_share_a_workspace():
    cases = [attention_case(shape(4, 2, 128), [500, 20, 300], [1, 60, 4], 100, 4, seed=1), attention_case(shape(4, 1, 128), [900], [1], 0, 0, seed=2),
             attention_case(shape(4, 2, 128, "fp32"), [90, 300], [50, 1], 0, 0, seed=3), attention_case(shape(8, 2, 64), [2000, 5], [2, 2], 0, 0, seed=4)]
    want = [run_attention(c) for c in cases]
    ws = torch.empty(max(B.blink_window_attention_workspace(c["m"], 60) for c in cases), dtype=torch.uint8, device="cuda")
    got = [run_attention(cases[i % 4], workspace=ws) for i in range(80)]
    assert all(torch.equal(g, want[i % 4]) for i, g in enumerate(got))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attention_a_query_that_is_no_number_stays_with_its_row(dtype, bad):
    for new in (1, 5, 90):
        c = attention_case(shape(4, 2, 64, dtype), [300, 30, 7], [new, new, 1], 50, 4, seed=new)
        rows = [new - 1, new]                              # the first request's last row, the second's first
        c["q"][rows] = 0
        out = run_attention(c)
        c["q"][rows, 3::64] = bad
        other = run_attention(c)
        assert not torch.isfinite(other[rows]).any()
        c["q"][rows], other[rows] = 0, out[rows]
        check_attention(c, other)


def test_attention_and_rotation_far_into_a_large_pool():
    """Blocks whose elements are more than 2^31, and their bytes more than 2^32, behind the pool's first."""
    blocks = 140_000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    for new in (1, 4, 70):
        c = attention_case(shape(4, 8, 128, layers=1), [200, 30, 0], [new, 1, new], 0, 0, seed=new, layer=0)
        small = c["pool"].shape[2]
        pool = torch.empty(1, 2, blocks, 8, BS, 128, dtype=torch.bfloat16, device="cuda")
        pool[:, :, blocks - small:] = c["pool"]
        c["table"] = torch.where((c["table"] >= 0) & (c["table"] < small), c["table"] + (blocks - small), c["table"])
        want = run_attention(c | {"table": torch.where(c["table"] >= blocks - small, c["table"] - (blocks - small), -1)})
        c["pool"] = pool
        assert torch.equal(run_attention(c), want)
    m, n = c["m"], 40
    x = torch.randn(n, m.qkv_dim, device="cuda").bfloat16()
    slots = blocks * BS - 1 - torch.randperm(n, device="cuda", dtype=torch.int32)
    B.blink_qk_norm_rope(m, pool, 0, x, None, None, ints(np.zeros(n)), slots)       # position 0: as they are
    heads = x[:, m.q_dim:].reshape(n, 2, 8, 128)
    for i in (0, 1):
        assert torch.equal(pool[0, i][slots.long() // BS, :, slots.long() % BS], heads[:, i])


def test_attention_max_new_is_a_hint():
    c = attention_case(shape(4, 2, 128), [90, 20, 300], [1, 90, 6], 64, 4, seed=5)
    for hint in (1, 2, 5, 90, 10000):
        check_attention(c, run_attention(c, max_new=hint))


def test_attention_many_requests():
    rng = np.random.default_rng(8)
    c = attention_case(shape(4, 1, 64), rng.integers(0, 60, 4096), (rng.random(4096) < 0.7).astype(int), 24, 2, seed=6)
    out = run_attention(c)
    check_attention(c, out, only=[0, 1, 2, 100, 2000, 4000, 4094, 4095])
    some = rng.permutation(4096)[:200]
    check_attention(c, out, only=some)


# ---- verification -----------------------------------------------------------------------------------------------------
def verify_case(rng, k, V, probs, temps, spread=2.0, stride=0):
    n, rows = len(k), int(np.sum(k)) + len(k)
    z = (spread * rng.normal(size=(rows, V + stride))).astype(np.float32)
    T = np.asarray(temps, np.float32)
    start = np.concatenate([[0], np.cumsum(np.asarray(k) + 1)])
    q = np.stack([O.target_probs(z[i, :V] + 0.5 * rng.normal(size=V), 1.0 if T[r] == 0 else T[r])[0] for r in range(n) for i in range(start[r], start[r + 1])])
    draft = np.array([rng.choice(V, p=x / x.sum()) for x in q])
    for r in range(n):
        if T[r] == 0:
            for i in range(start[r], start[r + 1]):
                if rng.random() < 0.8:
                    draft[i] = int(z[i, :V].argmax())
    return dict(z=z, V=V, start=start, draft=draft, q=q.astype(np.float32) if probs else None, T=T, ua=rng.random(rows).astype(np.float32),
                up=rng.random(n).astype(np.float32))


def run_verify(c, **kw):
    z = torch.from_numpy(c["z"]).cuda()[:, :c["V"]]
    f = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return B.blink_verify_drafts(z, ints(c["start"]), ints(c["draft"]), f(c["q"]) if c["q"] is not None else None, f(c["T"]), f(c["ua"]), f(c["up"]), **kw)


def check_verify(c, tokens, accepted):
    tokens, accepted = tokens.cpu().numpy(), accepted.cpu().numpy()
    for r in range(len(c["T"])):
        a, b = c["start"][r], c["start"][r + 1]
        if a == b:
            assert accepted[r] == 0
            continue
        want, n, near = O.verify_request(c["z"][a:b, :c["V"]], c["draft"][a:b - 1], None if c["q"] is None else c["q"][a:b], c["T"][r], c["ua"][a:b], c["up"][r])
        # a decision within 1e-7 (acceptance: the sum of 32-bit exponentials; the draw itself is good to 1e-13) is anybody's
        if near > 1e-7:
            assert accepted[r] == n and np.array_equal(tokens[a:b], want), (r, n, accepted[r], want, tokens[a:b], near)


@pytest.mark.parametrize("V", [2, 31, 257, 1000, 4096, 4097, 32000, 50001])
@pytest.mark.parametrize("probs", [True, False])
def test_verify(V, probs):
    rng = np.random.default_rng(V)
    k = [0, 1, 4, 7, 2, 0, 3, 5]
    c = verify_case(rng, k, V, probs, [1.0, 0.7, 0.0, 0.9, 1.3, 0.0, 0.05, 2.0], stride=V % 3)
    check_verify(c, *run_verify(c))


def test_verify_the_largest_vocabulary_of_the_configurations_and_one_beyond_shared_memory():
    rng = np.random.default_rng(1)
    for V in (128256, 210001):
        c = verify_case(rng, [3, 0, 6], V, True, [0.8, 1.0, 0.9], spread=1.5)
        check_verify(c, *run_verify(c))


def test_verify_many_draws_of_flat_rows():
    """Rows whose neighbours are as close as they come: the draw has to find the right one of some thousand."""
    rng = np.random.default_rng(2)
    c = verify_case(rng, [1] * 150, 5000, True, [1.0] * 150, spread=0.05)
    check_verify(c, *run_verify(c))


def test_verify_long_drafts():
    rng = np.random.default_rng(5)
    c = verify_case(rng, [150, 3], 600, True, [1.0, 0.9])
    c["ua"] *= 0.01                          # most are accepted
    check_verify(c, *run_verify(c))


def test_verify_the_same_call_gives_the_same_tokens():
    rng = np.random.default_rng(6)
    c = verify_case(rng, [3] * 40, 9000, True, [1.0] * 40, spread=0.1)
    first = run_verify(c)
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(first, run_verify(c)))


@pytest.mark.parametrize("V,probs", [(700, False), (40000, True), (70000, True), (150000, False)])
def test_verify_in_one_call_or_several_and_over_the_drafts(V, probs):
    rng = np.random.default_rng(V)
    k = [3, 0, 5, 1] * 7
    c = verify_case(rng, k, V, probs, [1.0, 0.0, 0.8, 1.1] * 7, spread=1.0)
    tokens, accepted = run_verify(c)
    check_verify(c, tokens, accepted)
    for a, b in ((0, 4), (4, 16), (16, 28)):
        s = slice(c["start"][a], c["start"][b])
        part = dict(c, z=c["z"][s], start=c["start"][a:b + 1] - c["start"][a], draft=c["draft"][s], q=c["q"][s] if probs else None, T=c["T"][a:b], ua=c["ua"][s], up=c["up"][a:b])
        some, n = run_verify(part)
        assert torch.equal(some, tokens[s]) and torch.equal(n, accepted[a:b])
        z = torch.from_numpy(part["z"]).cuda()
        f = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
        drafts = ints(part["draft"])
        B.blink_verify_drafts(z, ints(part["start"]), drafts, f(part["q"]) if probs else None, f(part["T"]), f(part["ua"]), f(part["up"]), out_tokens=drafts)
        assert torch.equal(drafts, some)


def test_verify_special_entries():
    rng = np.random.default_rng(3)
    V, n = 300, 12
    c = verify_case(rng, [2] * n, V, True, [0.9] * n)
    z, q, s = c["z"], c["q"], c["start"]
    z[s[0], :] = -np.inf                     # no number: greedy, token 0
    z[s[1], 50:] = np.nan                    # counts as -inf
    z[s[2], 7] = z[s[2], 9] = np.inf         # greedy, the first of them
    c["draft"][s[2]] = 7
    c["draft"][s[3]] = -1                    # outside the vocabulary
    c["draft"][s[4]] = V
    q[s[5]] = 2.0                            # q covers p: from p itself
    c["ua"][s[5]] = 0.99
    q[s[6], :100] = np.nan
    q[s[6], 100:200] = -1.0
    c["ua"][s[6]] = 1e9
    c["up"][7] = 1.5                         # past the end: the last with any weight
    c["up"][8], c["up"][9], c["up"][10] = 0.0, np.nan, -3.0
    c["T"][11] = np.inf
    c["ua"][s[9]] = np.nan
    z[s[10]:s[11], 100:] = -np.inf           # most of the row without weight
    check_verify(c, *run_verify(c))


def test_verify_temperatures_at_the_ends_of_their_range():
    step = 2.0 ** -19   # between neighbours at 22
    low = np.zeros(1000, np.float32)
    low[100:400] = np.float32(22 - 4 * step)   # exp(-790): nothing, and below what a 64-bit exponent holds
    low[5] = 22.0
    wide = np.zeros(1000, np.float32)
    wide[0] = -3.4e38                          # exp(-3.4) of the others' weight
    c = dict(z=np.stack([low, low, low, wide, wide]), V=1000, start=np.array([0, 1, 3, 4, 5]), draft=np.array([0, 5, 0, 0, 0]), q=None,
             T=np.array([4 * step / 790, 4 * step / 790, 1e38, 1e38], np.float32), ua=np.full(5, 0.5, np.float32),
             up=np.array([0.5, 0.999, 1e-5, 1e-4], np.float32))
    tokens, accepted = run_verify(c)
    check_verify(c, tokens, accepted)
    assert tokens.tolist() == [5, 5, 5, 0, 1] and accepted.tolist() == [0, 1, 0, 0]


def test_verify_rows_behind_the_last_request_and_requests_without_rows():
    rng = np.random.default_rng(4)
    c = verify_case(rng, [2, 3, 1, 2], 500, True, [1.0, 0.8, 0.7, 0.9])
    c["start"] = np.array([0, 3, 3, 7, 9])           # the second has none; two rows behind the last
    tokens = torch.full((c["z"].shape[0],), 77, dtype=torch.int32, device="cuda")
    out = run_verify(c, out_tokens=tokens)
    assert out[0] is tokens and (tokens[9:] == 77).all()
    check_verify(c, *out)


# ---- together, streams, graphs ----------------------------------------------------------------------------------------
def spec_step(m, st, stream_safe=True):
    """One step of all of them, as a program takes it; everything in st is on the device."""
    t = B.blink_build_tables(st["ctx"], st["new"], st["tables"].blocks_held, st["free"], st["tables"].free_count, st["table"], out=st["tables"])
    B.blink_qk_norm_rope(m, st["pool"], 0, st["qkv"], st["qg"], st["kg"], t.positions, t.slot_map, out=st["q"])
    B.blink_window_attention(m, st["pool"], 0, st["q"], t.row_start, t.kv_len, st["table"], st["window"], st["sinks"], st["max_new"], out=st["o"], workspace=st["ws"])
    st["logits"] = torch.matmul(st["o"].float(), st["head"], out=st["logits"])
    B.blink_verify_drafts(st["logits"], t.row_start, st["draft"], None, st["T"], st["ua"], st["up"], out_tokens=st["tok"], n_accepted=st["acc"], workspace=st["ws2"])


def spec_state(m, n, max_new, V=500, blocks=200, window=40, sinks=2, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = n * max_new
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)
    dt = DT[m.dtype]
    return dict(ctx=torch.zeros(n, dtype=torch.int32, device="cuda"), new=torch.full((n,), max_new, dtype=torch.int32, device="cuda"),
                tables=B.make_step_tables(n, rows, "cuda")._replace(free_count=ints([blocks])), free=ints(np.random.default_rng(seed).permutation(blocks)),
                table=torch.full((n, 24), -1, dtype=torch.int32, device="cuda"), pool=new_pool(m, blocks), qkv=r(rows, m.qkv_dim).to(dt),
                qg=1 + 0.1 * r(m.head_dim), kg=1 + 0.1 * r(m.head_dim), q=torch.zeros(rows, m.q_dim, dtype=dt, device="cuda"),
                o=torch.zeros(rows, m.q_dim, dtype=dt, device="cuda"), head=r(m.q_dim, V), logits=torch.zeros(rows, V, device="cuda"),
                draft=torch.zeros(rows, dtype=torch.int32, device="cuda"), T=torch.zeros(n, device="cuda"), ua=torch.rand(rows, device="cuda", generator=g),
                up=torch.rand(n, device="cuda", generator=g), tok=torch.zeros(rows, dtype=torch.int32, device="cuda"),
                acc=torch.zeros(n, dtype=torch.int32, device="cuda"), max_new=max_new, window=window, sinks=sinks, V=V,
                ws=torch.empty(B.blink_window_attention_workspace(m, max_new), dtype=torch.uint8, device="cuda"),
                ws2=torch.empty(B.blink_verify_workspace(rows, n, V), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_run_of_steps_is_the_same_captured_and_eager_and_follows_the_oracle(dtype):
    """Prompts, then drafts of one to four rows a request; lengths change from step to step under one graph, tokens that are refused are
    forgotten and their blocks used again."""
    m = shape(4, 2, 64, dtype, layers=1)
    n, most = 5, 30
    states = [spec_state(m, n, most), spec_state(m, n, most)]
    spec_step(m, states[1])                                    # (once outside the capture: modules are loaded)
    states[1] = spec_state(m, n, most)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        spec_step(m, states[1])
    torch.cuda.synchronize()
    history = [[] for _ in range(n)]                           # (k, v) of a request's tokens, in 64 bits, as cached
    for step in range(8):
        rng = np.random.default_rng(step)
        new = np.array([30, 17, 1, 0, 25]) if step == 0 else rng.integers(0, 5, n)
        ctx = np.array([len(h) for h in history])
        g = torch.Generator(device="cuda").manual_seed(100 + step)
        qkv = torch.randn(n * most, m.qkv_dim, device="cuda", generator=g).to(DT[dtype])
        draft = torch.randint(0, 500, (n * most,), device="cuda", generator=g, dtype=torch.int32)
        for st in states:
            st["ctx"].copy_(ints(ctx)); st["new"].copy_(ints(new)); st["qkv"].copy_(qkv); st["draft"].copy_(draft)
        torch.cuda.synchronize()
        spec_step(m, states[0])
        graph.replay()
        torch.cuda.synchronize()
        a, b = states
        for key in ("tok", "acc", "o", "table", "q"):
            assert torch.equal(a[key], b[key]), (step, key)
        assert all(torch.equal(x, y) for x, y in zip(a["tables"], b["tables"])) and int(a["tables"].status) == 0
        start = np.concatenate([[0], np.cumsum(new)])
        # the cache as the kernels left it is the oracle's input; every row's attention and verification follows from it
        slots, o = a["tables"].slot_map.cpu().numpy(), f64(a["o"])
        flat = [f64(a["pool"][0, i]).transpose(0, 2, 1, 3).reshape(-1, m.n_kv_heads, m.head_dim) for i in (0, 1)]
        case = dict(m=m, q=a["q"], start=start, ctx=ctx, window=40, sinks=2, kv=[])
        acc, tok = a["acc"].cpu().numpy(), a["tok"].cpu().numpy()
        for r in range(n):
            h = history[r] + [(flat[0][s], flat[1][s]) for s in slots[start[r]:start[r + 1]]]
            case["kv"].append(np.stack([np.stack([x[i] for x in h]) if h else np.zeros((0, m.n_kv_heads, m.head_dim)) for i in (0, 1)]))
            if new[r]:
                z = a["logits"][start[r]:start[r + 1]].cpu().numpy()
                want, k, _ = O.verify_request(z, draft[start[r]:start[r + 1] - 1].cpu().numpy(), None, 0.0, np.zeros(most), 0.0)
                assert acc[r] == k and np.array_equal(tok[start[r]:start[r + 1]], want)
            history[r] = h if step == 0 else h[:len(history[r]) + (int(acc[r]) + 1 if new[r] else 0)]
        check_attention(case, a["o"])
        held = a["tables"].blocks_held.cpu().numpy()
        table = a["table"].cpu().numpy()
        owned = np.concatenate([table[r, :held[r]] for r in range(n)])
        assert len(set(owned)) == len(owned) and int(a["tables"].free_count) + len(owned) == 200


def test_other_streams_than_the_default_one():
    m = shape(4, 2, 128)
    c = attention_case(m, [300, 20], [1, 60], 100, 4, seed=9)
    want = run_attention(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c["q"].mul_(1.0)
        got = [run_attention(c) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(want, g) for g in got)


def test_the_binding_refuses_what_does_not_fit():
    m = shape(4, 2, 128)
    c = attention_case(m, [20, 3], [1, 2], 0, 0)
    args = (c["m"], c["pool"], 0, c["q"], c["row_start"], c["kv_len"], c["table"], 0, 0, 2)

    def swap(i, x):
        return args[:i] + (x,) + args[i + 1:]
    for bad in (swap(3, c["q"].float()), swap(3, c["q"][:, :-8]), swap(4, c["row_start"][:-1]), swap(5, c["kv_len"].long()), swap(6, c["table"][:1])):
        with pytest.raises(ValueError):
            B.blink_window_attention(*bad)
    for bad in (swap(2, 2), swap(7, -1), swap(9, 0)):
        with pytest.raises(B.BlinkError) as e:
            B.blink_window_attention(*bad)
        assert e.value.code == B.BLINK_EINVAL
    with pytest.raises(B.BlinkError):
        B.blink_window_attention(*args, workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        B.blink_window_attention(*args, out=c["q"][:1].clone())


# ---- vocabularies that a draw goes over in several tiles --------------------------------------------------------------
@pytest.mark.parametrize("V", [131073, 150000, 393217])
def test_verify_refused_drafts_of_a_vocabulary_of_several_tiles(V):
    """The token comes from p - q, tile by tile: each with its own q."""
    rng = np.random.default_rng(V)
    k = [2, 1, 3]
    c = verify_case(rng, k, V, True, [1.0, 0.8, 1.2], spread=1.0)
    c["ua"][:] = 1e9                         # the first draft of each is refused
    tokens, accepted = run_verify(c)
    assert accepted.tolist() == [0, 0, 0]
    check_verify(c, tokens, accepted)
    for _ in range(10):
        assert torch.equal(run_verify(c)[0], tokens)


# ---- a long run of short units ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("rep,hkv,hd,window", [(4, 8, 64, 0), (8, 2, 128, 0), (4, 4, 128, 9)])
def test_attention_runs_of_short_units_and_long_ones_among_them(rep, hkv, hd, window):
    """Many units of one tile of keys a CTA, with rows for one stream only: the other one passes them by."""
    rng = np.random.default_rng(hd + rep)
    n = 3000
    new = rng.integers(2, 5, n)
    new[::97] = 300                          # two streams, several tiles
    c = attention_case(shape(rep, hkv, hd, layers=1), rng.integers(0, 60, n), new, window, 1, seed=n, layer=0)
    out = run_attention(c)
    check_attention(c, out, only=[0, 1, 2, 96, 97, 98] + rng.permutation(n)[:60].tolist())
    for _ in range(5):
        assert torch.equal(run_attention(c), out)


# ---- launches ---------------------------------------------------------------------------------------------------------
def fresh_process(code):
    """Runs code in a process of its own (the state of a kernel's attributes outlives a call); it prints nothing when it is right."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", "import sys; sys.path[:0] = [%r, %r]\n" % (root, os.path.join(root, "tests")) + code], capture_output=True, text=True,
                       timeout=300, cwd=root)
    assert r.returncode == 0 and r.stdout == "", r.stdout + r.stderr


def test_tables_where_dynamic_and_static_shared_memory_reach_48_kb_together():
    fresh_process("""
import numpy as np
from test_gpu_step import check_tables, tables_case
for n in (3037, 3038, 3039, 3055, 3070, 3071):
    check_tables(*tables_case(np.random.default_rng(n), n, 20, 2, 3))
""")


@pytest.mark.parametrize("hd,sizes", [(128, (1996, 1997, 1998, 1999, 2000)), (64, (2508, 2509, 2510, 2511, 2512))])
def test_attention_where_dynamic_and_static_shared_memory_reach_48_kb_together(hd, sizes):
    fresh_process(f"""
import numpy as np
from test_gpu_step import attention_case, check_attention, run_attention, shape
for n in {sizes}:
    c = attention_case(shape(1, 1, {hd}, layers=1), np.random.default_rng(n).integers(1, 90, n), [1] * n, 0, 0, seed=n, layer=0)
    check_attention(c, run_attention(c), only=[0, 1, n // 2, n - 1])
""")


def in_two_threads(calls, times=2000):
    """Both calls again and again, each by a host thread with a stream of its own (ctypes lets go of the interpreter); the codes other
    than BLINK_OK."""
    import threading
    bad, gate = [], threading.Barrier(len(calls))

    def loop(call):
        stream = torch.cuda.Stream()
        gate.wait()
        for i in range(times):
            rc = call(stream.cuda_stream)
            if rc != B.BLINK_OK:
                bad.append(rc)
            if i % 100 == 99:
                stream.synchronize()
    threads = [threading.Thread(target=loop, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return bad


def test_tables_of_different_sizes_from_two_host_threads():
    def caller(n):
        rows = 64
        zero, one = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        out = B.make_step_tables(n, rows, "cuda")
        table = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
        p = lambda t: t.data_ptr()
        return lambda stream, keep=(zero, one, out, table): B.lib().blink_build_tables(
            p(zero), p(zero), p(zero), n, p(one), 1, p(one), p(table), 1, rows, p(out.blocks_held), p(out.free_count), p(out.row_start), p(out.kv_len),
            p(out.positions), p(out.slot_map), p(out.status), stream)
    calls = [caller(4096), caller(3200)]
    torch.cuda.synchronize()
    assert in_two_threads(calls, 20000) == []


def test_attention_of_different_sizes_from_two_host_threads():
    import ctypes as C

    def caller(n, new):
        c = attention_case(shape(4, 1, 128, layers=1), [5] * n, [new] * n, 0, 0, seed=n, layer=0)
        cfg = B.make_model_cfg(c["m"])
        kv = B.blink_kv_pool(C.sizeof(B.blink_kv_pool), 16, c["pool"].data_ptr(), c["pool"].numel() * 2)
        out, ws = torch.zeros_like(c["q"]), torch.zeros(B.blink_window_attention_workspace(c["m"], new), dtype=torch.uint8, device="cuda")
        p = lambda t: t.data_ptr()
        return (lambda stream: B.lib().blink_window_attention(C.byref(cfg), C.byref(kv), 0, p(c["q"]), 512, n * new, p(c["row_start"]), p(c["kv_len"]), n, p(c["table"]),
                                                              c["table"].shape[1], 0, 0, new, p(out), 512, p(ws), ws.numel(), stream)), c, out
    many, few = caller(300, 9), caller(2, 9)
    torch.cuda.synchronize()
    assert in_two_threads([many[0], few[0]], 500) == []
    for _, c, out in (many, few):
        check_attention(c, out, only=[0, 1])


@pytest.mark.parametrize("dtype,new", [("bf16", 9), ("bf16", 1), ("fp32", 9)])
def test_attention_from_a_host_thread_that_has_not_used_the_device(dtype, new):
    import threading
    c = attention_case(shape(4, 2, 128, dtype), [50, 3], [new, 1], 0, 0)
    want, out = run_attention(c), torch.zeros_like(c["q"])
    ws = torch.zeros(B.blink_window_attention_workspace(c["m"], new), dtype=torch.uint8, device="cuda")
    failed = []

    def call():
        try:
            run_attention(c, out=out, workspace=ws)
        except B.BlinkError as e:
            failed.append(e)
    torch.cuda.synchronize()
    t = threading.Thread(target=call)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert failed == [] and torch.equal(out, want)


@pytest.mark.parametrize("rep,hkv,hd,dtype", [(4, 2, 128, "bf16"), (8, 1, 64, "bf16"), (1, 2, 128, "bf16"), (4, 2, 64, "fp32")])
def test_attention_a_workspace_for_long_requests_serves_shorter_ones(rep, hkv, hd, dtype):
    m = shape(rep, hkv, hd, dtype)
    ws = torch.empty(B.blink_window_attention_workspace(m, 4096), dtype=torch.uint8, device="cuda")
    for new in (1, 2, 3, 4, 5, 6, 7, 8, 9, 13, 29, 32, 33):
        c = attention_case(m, [40, 3, 900], [new, 1, new], 0, 0, seed=new)
        check_attention(c, run_attention(c, workspace=ws))


# ---- temperatures -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("V", [50, 5000, 40000, 100000])
@pytest.mark.parametrize("T", [1e-6, 1e-12, 1e-18, 1e-20, 1e-30, 1.2e-38])
def test_verify_small_temperatures_share_a_row_among_its_largest(T, V):
    """Largest entries that are no short binary fractions, twice in a row: half the weight each, whatever the temperature."""
    rng = np.random.default_rng(int(-np.log10(T)) * 7 + V)
    n = 40
    z = (rng.normal(size=(2 * n, V)) * 2).astype(np.float32)
    a, b = rng.permutation(V)[:2 * n].reshape(2, n) if V >= 2 * n else (np.arange(n) % 25, 25 + np.arange(n) % 25)
    for r in range(n):
        z[2 * r:2 * r + 2, [a[r], b[r]]] = np.float32(5 + 25 * rng.random())
    draft = np.zeros(2 * n, np.int64)
    draft[::2] = a
    c = dict(z=z, V=V, start=2 * np.arange(n + 1), draft=draft, q=None, T=np.full(n, T, np.float32), ua=np.tile(np.float32([0.4, 0.0, 0.6, 0.0]), n // 2),
             up=rng.random(n).astype(np.float32))
    tokens, accepted = run_verify(c)
    check_verify(c, tokens, accepted)
    planted = z[2 * np.arange(n), a] == z.reshape(n, 2 * V).max(1)                  # (in some rows another entry came out larger)
    odd = np.arange(n) % 2 == 1
    assert planted.sum() > 20 and np.array_equal(accepted.cpu().numpy()[planted], 1 - odd[planted])
    want = np.where(odd, b, np.where(c["up"] < 0.5, np.minimum(a, b), np.maximum(a, b)))   # refused: the other one; else either half
    tokens = tokens.cpu().numpy().reshape(n, 2)
    assert np.array_equal(np.where(odd, tokens[:, 0], tokens[:, 1])[planted], want[planted])


def test_verify_the_ends_of_the_temperatures_range_in_the_acceptance():
    """Differences of entries beyond 32 bits at temperatures as large, and entries a few smallest numbers apart at temperatures as small: a draft is
    accepted with the probability that these give it."""
    rows, T = [], []
    for V in (60, 5000):
        for t, lo, hi in ((3.4e38, -3.4e38, 3.4e38), (1e37, 3.35e38, 3.4e38), (2e30, -1e30, 3e30), (1e-45, -3e-45, 0.0), (3e-39, 0.0, 5e-39), (1e-40, -2e-40, 1e-40),
                          (1e-38, -0.5, 0.5), (1e-38, -3e38, 0.9), (1e-44, 1.5, 1.5)):
            z = np.full(V, lo, np.float32)
            z[V // 3::7] = hi
            z[V // 2] = -np.inf
            rows += [z, z]
            T.append(t)
    n = len(T)
    for V in (60, 5000):
        sel = [i for i in range(n) if len(rows[2 * i]) == V]
        for high in (0, 1):                    # the draft is one of the low, or of the high entries
            z = np.stack([r for i in sel for r in rows[2 * i:2 * i + 2]])
            x = V // 3 + (0 if high else 1)
            T32 = np.array([T[i] for i in sel], np.float32)
            p = np.array([O.target_probs(z[2 * i], T32[i])[0][x] for i in range(len(sel))])
            for f in (0.97, 1.03):
                ua = np.zeros(2 * len(sel), np.float32)
                ua[::2] = p * f
                c = dict(z=z, V=V, start=2 * np.arange(len(sel) + 1), draft=np.full(2 * len(sel), x), q=None, T=T32, ua=ua, up=np.full(len(sel), 0.37, np.float32))
                tokens, accepted = run_verify(c)
                check_verify(c, tokens, accepted)
                some = p > 1e-30
                assert some.any() and np.array_equal(accepted.cpu().numpy()[some], np.full(some.sum(), int(f < 1)))


def test_an_error_of_another_call_is_not_the_operators():
    """A loop that is refused for want of memory leaves an error behind in the library; the operators' launches succeed all the same, all
    of a call's kernels."""
    import ctypes as C
    m = shape(4, 2, 128)
    cfg = B.make_model_cfg(m)
    sched = B.blink_sched_cfg(size=C.sizeof(B.blink_sched_cfg), max_batch=8, prefill_chunk_tokens=64, n_slots=1024, max_prompt=1 << 30, max_new=16, control_only=1)
    kv = B.blink_kv_pool(C.sizeof(B.blink_kv_pool), 16, None, 64 * B.kv_bytes_per_block(m))
    c = attention_case(m, [30000, 3], [1, 1], 0, 0)                       # two kernels
    v = verify_case(np.random.default_rng(0), [3] * 14, 500, True, [0.9] * 14)   # three
    want, wv = run_attention(c), run_verify(v)

    def refused():
        ctx = C.c_void_p()
        assert B.lib().blink_create(C.byref(cfg), C.byref(sched), C.byref(kv), C.byref(ctx)) == B.BLINK_ENOMEM    # 4 TB of prompts
    refused()
    assert torch.equal(run_attention(c), want)
    refused()
    assert all(torch.equal(x, y) for x, y in zip(run_verify(v), wv))


def test_the_binding_takes_a_pool_of_the_models_type_and_shape_or_bytes():
    for dtype, other in (("bf16", torch.float32), ("bf16", torch.float16), ("fp32", torch.bfloat16)):
        m = shape(4, 2, 128, dtype)
        c = attention_case(m, [20, 3], [1, 2], 0, 0)
        want, pool = run_attention(c), c["pool"]
        assert torch.equal(run_attention(c | {"pool": pool.view(torch.uint8)}), want) and torch.equal(run_attention(c | {"pool": pool.view(-1).view(torch.uint8)}), want) and torch.equal(run_attention(c | {"pool": pool.view(-1)}), want)
        x = torch.zeros(3, m.qkv_dim, dtype=DT[dtype], device="cuda")
        for bad in (pool.to(other), pool.view(-1).to(other), pool[:1], pool[:, :, :, :1].contiguous(), pool[..., :64].contiguous(), pool.transpose(3, 4).contiguous(),
                    pool.transpose(0, 2)):
            with pytest.raises(ValueError, match="kv_pool"):
                run_attention(c | {"pool": bad})
            with pytest.raises(ValueError, match="kv_pool"):
                B.blink_qk_norm_rope(m, bad, 0, x, None, None, ints([0, 1, 2]), ints([0, 1, 2]))


def test_rows_that_belong_to_nobody_are_defined_in_outputs_that_the_binding_makes():
    """Memory that was used before, as a captured step with spare rows would read it on: zeros, and tokens of -1."""
    def dirty(*shape_of, dtype):
        t = [torch.full(shape_of, 7 if dtype == torch.int32 else float("nan"), dtype=dtype, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        del t
    for dtype in ("bf16", "fp32"):
        m = shape(4, 2, 128, dtype)
        c = attention_case(m, [50, 3], [3, 40], 0, 0, pad=9)
        dirty(*c["q"].shape, dtype=DT[dtype])
        out = run_attention(c)
        check_attention(c, out)
        assert (out[43:] == 0).all()
        x = torch.randn(30, m.qkv_dim, device="cuda").to(DT[dtype])
        dirty(30, m.q_dim, dtype=DT[dtype])
        q = B.blink_qk_norm_rope(m, new_pool(m, 3), 0, x, None, None, ints([1] * 20 + [-1] * 10), ints([-1] * 30))
        assert (q[20:] == 0).all() and (q[:20] != 0).any()
    for n in (3, 20):                       # two kernels, three
        v = verify_case(np.random.default_rng(n), [2] * n, 3000, True, [0.9] * n)
        v["start"] = v["start"][:-1]
        v["T"], v["up"] = v["T"][:-1], v["up"][:-1]
        dirty(3 * n, dtype=torch.int32)
        tokens, accepted = run_verify(v)
        check_verify(v, tokens, accepted)
        assert (tokens[3 * n - 3:] == -1).all()
        kept = torch.full((3 * n,), 77, dtype=torch.int32, device="cuda")
        assert (run_verify(v, out_tokens=kept)[0][3 * n - 3:] == 77).all() and torch.equal(kept[:3 * n - 3], tokens[:3 * n - 3])
