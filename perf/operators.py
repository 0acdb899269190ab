"""Operators of one speculative decoding step over the paged KV cache, and the cases by which their speed is judged.

A step with drafted tokens, as a serving program takes it beside the loop: the requests' lengths become block tables and a slot
map ("tables"); the projected queries and keys are normed per head, rotated, and the keys and values cached ("norm_rope"); the new
rows attend over the cache, through a sliding window and a few first tokens that stay visible ("attention"); and the drafted tokens are held
against the target's probabilities ("verify").

The pool has the layout of the serving loop, [layers][2][blocks][kv heads][16 tokens][head_dim]; model shapes are the
small, the 1B and the 8B configuration of the repository.  `run` computes an operator from elementary operations, or through the
framework where `own` is true; `exact` computes it once more from its definition in 64 bits.
"""
import math
import random
from dataclasses import dataclass

import numpy as np
import torch

own = False

BS = 16   # tokens of a block


@dataclass(frozen=True)
class Shape:
    n_layers: int
    d_model: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    d_ff: int
    vocab: int
    rope_theta: float
    dtype: str
    n_experts: int = 0
    top_k_experts: int = 0
    rms_eps: float = 1e-5


def _shape(case):
    """One or two layers of a configuration (a cache of all of them would not fit several times; a call handles one layer)."""
    args = {"tiny": (256, 4, 4, 64, 1024, 4096, 1e4), "1b": (2048, 32, 8, 64, 8192, 32000, 1e4), "8b": (4096, 32, 8, 128, 14336, 128256, 5e5)}[case["model"]]
    return Shape(case["layers"], *args, case["dtype"])


# ---- cases ------------------------------------------------------------------------------------------------------
def _tables(name, requests, ctx, new, spare):
    c = dict(op="tables", requests=requests, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1], spare=spare)
    return dict(name=name, **c) if name else c


def _norm_rope(name, model, dtype, qkv, rows, first, norm=True):
    c = dict(op="norm_rope", model=model, layers=2, dtype=dtype, qkv=qkv, rows=rows, first=first, norm=norm)
    return dict(name=name, **c) if name else c


def _attention(name, model, dtype, requests, ctx, new, window, sinks):
    c = dict(op="attention", model=model, layers=1, dtype=dtype, requests=requests, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1],
             window=window, sinks=sinks)
    return dict(name=name, **c) if name else c


def _verify(name, vocab, requests, drafts, probs, greedy):
    c = dict(op="verify", vocab=vocab, requests=requests, drafts_lo=drafts[0], drafts_hi=drafts[1], probs=probs, greedy=greedy)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the batch of the small configuration decodes: one row each, hardly any new block; the smallest call, latency is all there is
        _tables("tables 8 decoding", 8, (4, 90), (1, 1), 0),
        # a full batch of the 8B configuration, chunks of long prompts and decode rows mixed; a graph's rows behind the last
        _tables("tables 256 mixed", 256, (0, 5000), (1, 1500), 517),
        # decode step of 64 conversations of the 8B shape
        _norm_rope("norm rope 8b 64 rows", "8b", "bf16", "bf16", 64, 4000),
        # a prompt of the 8B shape; projections left in 32 bits, as the loop's GEMMs leave them
        _norm_rope("norm rope 8b 4099 rows", "8b", "bf16", "fp32", 4099, 0),
        # a single user far into a conversation: one row, latency
        _attention("attention 8b one row", "8b", "bf16", 1, (4800, 4800), (1, 1), 1024, 4),
        # decode step of a large batch with contexts of all lengths
        _attention("attention 8b 200 rows", "8b", "bf16", 200, (20, 5000), (1, 1), 2048, 4),
        # rows of drafted tokens, to be verified: one to six a request
        _attention("attention 8b drafts", "8b", "bf16", 48, (300, 5000), (1, 6), 4096, 4),
        # whole prompts of the longest kind and rests of others
        _attention("attention 8b prompts", "8b", "bf16", 3, (0, 1000), (2000, 4096), 1024, 4),
        # head_dim 64: chunks of prompts beside decode rows
        _attention("attention 1b chunks", "1b", "bf16", 40, (0, 900), (1, 300), 256, 1),
        # the 32-bit reference mode: a batch of the small configuration with its prompts
        _attention("attention tiny fp32", "tiny", "fp32", 8, (0, 64), (16, 64), 48, 2),
        # a single user with a few drafts, probabilities of a draft model
        _verify("verify one request", 32000, 1, (4, 4), True, 0.0),
        # a batch of conversations with drafts of different lengths, some of them greedy
        _verify("verify 64 requests", 128256, 64, (0, 7), True, 0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(case):
    """Elements of the largest thing that a pass of the plain form makes."""
    if case["op"] == "tables":
        return _ctx_new(case)[1].sum()
    if case["op"] == "norm_rope":
        return case["rows"] * (_shape(case).n_q_heads + 2 * _shape(case).n_kv_heads) * _shape(case).head_dim
    if case["op"] == "verify":
        return (_drafts(case).sum() + case["requests"]) * case["vocab"]
    s, (ctx, new) = _shape(case), _ctx_new(case)
    seen = _columns(case)
    return case["requests"] * seen * (new.max() * s.n_q_heads + 2 * s.n_kv_heads * s.head_dim)


_MOST = {"tables": 110_000, "norm_rope": 4099 * 6144, "attention": 1_300_000_000, "verify": 300 * 128256}


def draw(rng):
    """One more case: an operator, and sizes anywhere in the ranges of the listed ones."""
    op = rng.choice(["tables", "norm_rope", "attention", "attention", "attention", "verify"])
    model = rng.choice(["tiny", "1b", "8b", "8b"])
    dtype = rng.choice(["bf16", "fp32"]) if model == "tiny" else "bf16"
    while True:
        if op == "tables":
            ctx, new = rng.randint(0, 300), _log_int(rng, 1, 700)
            c = _tables(None, _log_int(rng, 1, 256), (ctx, ctx + rng.randint(0, 4500)), (min(new, rng.choice([0, 1, 1, 20])), new), rng.choice([0, 0, rng.randint(1, 600)]))
        elif op == "norm_rope":
            c = _norm_rope(None, model, dtype, "fp32" if dtype == "fp32" else rng.choice(["bf16", "fp32"]), _log_int(rng, 1, 4000), rng.choice([0, rng.randint(1, 100000)]),
                           rng.choice([True, True, False]))
        elif op == "verify":
            k = rng.randint(0, 7)
            c = _verify(None, rng.choice([4096, 32000, 128256, rng.randint(1000, 128256)]), _log_int(rng, 1, 64), (rng.randint(0, k), k), rng.choice([True, True, False]),
                        rng.choice([0.0, 0.0, 0.3, 1.0]))
        else:
            long = {"tiny": 96, "1b": 1500, "8b": 5000}[model]
            ctx = _log_int(rng, 1, long)
            new = rng.choice([1, rng.randint(2, 8), _log_int(rng, 8, max(9, long * 3 // 4))])
            c = _attention(None, model, dtype, _log_int(rng, 1, 200), (rng.randint(0, ctx), ctx), (rng.randint(1, new), new), rng.choice([0, _log_int(rng, 16, 4096)]),
                           rng.choice([0, 1, 4, 4, rng.randint(5, 40)]))
        if _size(c) <= _MOST[op]:
            return c


# ---- lengths: they follow from the case alone, not from the seed ------------------------------------------------
def _spread(lo, hi, n, key):
    """n lengths, spread evenly over the logarithm of [lo, hi] (one half of them at least, where lo is 0), in a mixed order."""
    v = [int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** ((i + 0.5) / n))) - 1 for i in range(n)]
    random.Random(key).shuffle(v)
    return np.array([max(lo, min(hi, x)) for x in v], dtype=np.int64)


def _ctx_new(case):
    n = case["requests"]
    return _spread(case["ctx_lo"], case["ctx_hi"], n, 1), _spread(case["new_lo"], case["new_hi"], n, 2)


def _drafts(case):
    return _spread(case["drafts_lo"], case["drafts_hi"], case["requests"], 3)


def _first_seen(case):
    """First position behind the sinks that some row of the request sees."""
    ctx, _ = _ctx_new(case)
    return np.maximum(case["sinks"], ctx - case["window"] + 1) if case["window"] else np.minimum(case["sinks"], ctx)


def _columns(case):
    """Positions that the rows of a request see, at most: the sinks, and those from the first row's window on."""
    ctx, new = _ctx_new(case)
    return int(max(case["sinks"] + e - f for e, f in zip(ctx + new, _first_seen(case))))


def _pairs(case):
    """Pairs of a row and a position that it sees."""
    ctx, new = _ctx_new(case)
    total = 0
    for c, m in zip(ctx, new):
        p = np.arange(c, c + m)
        w = case["window"] or int(c + m)
        first = np.maximum(0, p - w + 1)
        total += int((p + 1 - first + np.minimum(first, case["sinks"])).sum())
    return total


def work(case):
    if case["op"] == "tables":
        ctx, new = _ctx_new(case)
        need = ((ctx + new + BS - 1) // BS - (ctx + BS - 1) // BS).sum()
        n = case["requests"]
        return {"bytes": float(4 * (3 * n + 1 + need) + 4 * (need + 3 * n + 3) + 8 * (new.sum() + case["spare"])), "flops": 0.0}
    if case["op"] == "verify":
        rows, n, V = int(_drafts(case).sum()) + case["requests"], case["requests"], case["vocab"]
        return {"bytes": float(4 * V * (rows + (n if case["probs"] else 0)) + 16 * rows + 16 * n), "flops": 3.0 * rows * V}
    s = _shape(case)
    e = 2 if s.dtype == "bf16" else 4
    if case["op"] == "norm_rope":
        el = case["rows"] * (s.n_q_heads + 2 * s.n_kv_heads) * s.head_dim
        return {"bytes": float(el * ((2 if case["qkv"] == "bf16" else 4) + e) + 8 * case["rows"]), "flops": 7.0 * el}
    ctx, new = _ctx_new(case)
    seen = (ctx + new - _first_seen(case) + np.minimum(case["sinks"], _first_seen(case))).sum()
    q = int(new.sum()) * s.n_q_heads * s.head_dim
    return {"bytes": float((2 * q + 2 * int(seen) * s.n_kv_heads * s.head_dim) * e), "flops": 4.0 * _pairs(case) * s.n_q_heads * s.head_dim}


# ---- inputs -----------------------------------------------------------------------------------------------------
def _torch(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _starts(new):
    return np.concatenate([[0], np.cumsum(new)])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    op = case["op"]
    st = dict(op=op)
    if op == "tables":
        ctx, new = _ctx_new(case)
        n, rows = len(ctx), int(new.sum()) + case["spare"]
        held = (ctx + BS - 1) // BS
        need = (ctx + new + BS - 1) // BS - held
        stride = int((held + need).max()) + 3
        ids = rng.permutation(int((held + need).sum()) + 40)
        table = np.full((n, stride), -1)
        at = 0
        for r in range(n):
            table[r, :held[r]] = ids[at:at + held[r]]
            at += held[r]
        st.update(ctx_len=_ints(ctx), new_len=_ints(new), blocks_held=_ints(held), free_blocks=_ints(ids[at:]), free_count=_ints([len(ids) - at]),
                  block_table=_ints(table), max_rows=rows)
        # what a program keeps from step to step: the operator's outputs
        st["out"] = tuple(torch.zeros(k, dtype=torch.int32, device="cuda") for k in (n + 1, n, rows, rows, n, 1, 1))
        return st
    if op == "verify":
        k, V = _drafts(case), case["vocab"]
        n, rows = len(k), int(k.sum()) + len(k)
        logits = torch.empty(rows, V, device="cuda").normal_(0, 2.0, generator=g)
        temperature = rng.uniform(0.6, 1.1, n).astype(np.float32)
        temperature[rng.random(n) < case["greedy"]] = 0.0
        T = torch.from_numpy(np.repeat(np.where(temperature > 0, temperature, 1.0), k + 1).astype(np.float32)).cuda()[:, None]
        # a draft model's probabilities: near the target's; drafts are drawn from them (greedy requests: mostly the largest)
        probs = torch.softmax(logits / T + torch.empty_like(logits).normal_(0, 0.6, generator=g), -1)
        tokens = torch.multinomial(probs, 1, generator=g)[:, 0]
        best = torch.from_numpy(np.repeat(temperature == 0, k + 1) & (rng.random(rows) < 0.8)).cuda()
        tokens = torch.where(best, logits.argmax(-1), tokens).to(torch.int32)
        st.update(logits=logits, row_start=_ints(_starts(k + 1)), draft_tokens=tokens, draft_probs=probs if case["probs"] else None,
                  temperature=torch.from_numpy(temperature).cuda(), u_accept=torch.rand(rows, device="cuda", generator=g),
                  u_pick=torch.rand(n, device="cuda", generator=g), longest=int(k.max()) + 1)
        return st
    s = _shape(case)
    st["model"], st["layer"] = s, s.n_layers - 1
    dt = _torch(s.dtype)
    if op == "norm_rope":
        rows = case["rows"]
        blocks = rows // BS + 40
        qkv = torch.empty(rows, (s.n_q_heads + 2 * s.n_kv_heads) * s.head_dim, device="cuda").normal_(0, 1.3, generator=g).to(_torch(case["qkv"]))
        gains = [torch.empty(s.head_dim, device="cuda").normal_(1, 0.2, generator=g) if case["norm"] else None for _ in range(2)]
        pool = torch.zeros(s.n_layers, 2, blocks, s.n_kv_heads, BS, s.head_dim, dtype=dt, device="cuda")
        # a prompt's rows follow one another in blocks from anywhere in the pool; rows of a decode step have positions of their own
        if case["first"]:
            positions, slots = rng.integers(0, case["first"], rows), rng.permutation(blocks * BS)[:rows]
        else:
            positions = np.arange(rows)
            slots = rng.permutation(blocks)[positions // BS] * BS + positions % BS
        st.update(qkv=qkv, q_gain=gains[0], k_gain=gains[1], pool=pool, positions=_ints(positions), slots=_ints(slots),
                  q_out=torch.zeros(rows, s.n_q_heads * s.head_dim, dtype=dt, device="cuda"))
        return st
    ctx, new = _ctx_new(case)
    n, rows = len(ctx), int(new.sum())
    first = _first_seen(case)
    have = (ctx + new + BS - 1) // BS
    used = [[b for b in range(have[r]) if b * BS < case["sinks"] or (b + 1) * BS > first[r]] for r in range(n)]
    total = sum(map(len, used))
    ids = rng.permutation(total + 24)
    table = np.full((n, int(have.max()) + 2), -1)   # blocks that nobody sees any more have been given back
    at = 0
    for r in range(n):
        table[r, used[r]] = ids[at:at + len(used[r])]
        at += len(used[r])
    pool = torch.empty(1, 2, total + 24, s.n_kv_heads, BS, s.head_dim, dtype=dt, device="cuda").normal_(0, 1, generator=g)
    q = torch.empty(rows, s.n_q_heads * s.head_dim, dtype=dt, device="cuda").normal_(0, 1.2, generator=g)
    st.update(pool=pool, q=q, row_start=_ints(_starts(new)), kv_len=_ints(ctx + new), table=_ints(table), window=case["window"], sinks=case["sinks"],
              max_new=int(new.max()), columns=_columns(case), out=torch.zeros_like(q))
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    return {"tables": _plain_tables, "norm_rope": _plain_norm_rope, "attention": _plain_attention, "verify": _plain_verify}[state["op"]](state)


def _run_own(st):
    from paper_2604_07609_b200 import binding as B
    if st["op"] == "tables":
        t = B.blink_build_tables(st["ctx_len"], st["new_len"], st["blocks_held"], st["free_blocks"], st["free_count"], st["block_table"], out=st["out"])
        return {"table": st["block_table"], "rest": list(t)}
    if st["op"] == "norm_rope":
        q = B.blink_qk_norm_rope(st["model"], st["pool"], st["layer"], st["qkv"], st["q_gain"], st["k_gain"], st["positions"], st["slots"], out=st["q_out"])
        return {"q": q, "kv": st["pool"][st["layer"]]}
    if st["op"] == "attention":
        return B.blink_window_attention(st["model"], st["pool"], st["layer"], st["q"], st["row_start"], st["kv_len"], st["table"], st["window"], st["sinks"],
                                        st["max_new"], out=st["out"])
    tokens, accepted = B.blink_verify_drafts(st["logits"], st["row_start"], st["draft_tokens"], st["draft_probs"], st["temperature"], st["u_accept"], st["u_pick"])
    return {"tokens": tokens, "accepted": accepted}


def _plain_tables(st):
    ctx, new, held, table = (st[k].long() for k in ("ctx_len", "new_len", "blocks_held", "block_table"))
    n, stride, rows = len(ctx), table.shape[1], st["max_rows"]
    need = ((ctx + new + BS - 1) // BS - held).clamp_(min=0)
    before = need.cumsum(0) - need
    j = torch.arange(stride, device="cuda")[None, :] - held[:, None]
    popped = st["free_count"].long() - 1 - (before[:, None] + j)
    fresh = st["free_blocks"].long()[popped.clamp(0, len(st["free_blocks"]) - 1)]
    table = torch.where((j >= 0) & (j < need[:, None]), fresh, table)
    ends = new.cumsum(0)
    row = torch.arange(rows, device="cuda")
    r = torch.searchsorted(ends, row, right=True).clamp_(max=n - 1)
    pos = ctx[r] + row - (ends - new)[r]
    slot = table[r, (pos // BS).clamp_(max=stride - 1)] * BS + pos % BS
    live = row < ends[-1]
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    rest = [torch.cat([zero, ends]), ctx + new, torch.where(live, pos, -1), torch.where(live, slot, -1), held + need, st["free_count"] - need.sum(), zero]
    return {"table": table.to(torch.int32), "rest": [x.to(torch.int32) for x in rest]}


def _plain_norm_rope(st):
    s, pool = st["model"], st["pool"][st["layer"]]
    Hq, Hkv, hd = s.n_q_heads, s.n_kv_heads, s.head_dim
    x = st["qkv"].float().view(-1, Hq + 2 * Hkv, hd)
    q, k, v = x.split([Hq, Hkv, Hkv], 1)
    if st["q_gain"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + s.rms_eps) * st["q_gain"]
        k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + s.rms_eps) * st["k_gain"]
    i = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
    angle = st["positions"].double()[:, None] * s.rope_theta ** (-2.0 * i / hd)
    c, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(y):
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * sn, b * c + a * sn], -1).to(pool.dtype)
    st["q_out"].copy_(turned(q).reshape(len(x), -1))
    block, at = st["slots"].long() // BS, st["slots"].long() % BS
    pool[0][block, :, at] = turned(k)
    pool[1][block, :, at] = v.to(pool.dtype)
    return {"q": st["q_out"], "kv": pool}


def _plain_attention(st):
    s, pool = st["model"], st["pool"][st["layer"]]
    Hkv, hd, rep = s.n_kv_heads, s.head_dim, s.n_q_heads // s.n_kv_heads
    start, kv_len, table = st["row_start"].long(), st["kv_len"].long(), st["table"].long()
    new = start[1:] - start[:-1]
    n, M, C, W, S = len(kv_len), st["max_new"], st["columns"], st["window"], st["sinks"]
    # the positions that a request's rows see: the sinks, then those from the first row's window on
    first = (kv_len - new - W + 1).clamp(min=S) if W else torch.clamp(kv_len - new, max=S)
    col = torch.arange(C, device="cuda")
    pos = torch.where(col < S, col, first[:, None] + col - S)
    there = (pos < kv_len[:, None]) & ((col >= S) | (pos < first[:, None]))
    block = table.gather(1, (pos // BS).clamp(max=table.shape[1] - 1)).clamp_(min=0)
    k, v = (pool[i][block, :, pos % BS].permute(0, 2, 1, 3).float() for i in (0, 1))   # [n, Hkv, C, hd]
    v = v * there[:, None, :, None]
    i = torch.arange(M, device="cuda")
    row = (start[:-1, None] + i).clamp_(max=len(st["q"]) - 1)
    q = st["q"][row].float().view(n, M, Hkv, rep, hd).permute(0, 2, 1, 3, 4).reshape(n, Hkv, M * rep, hd)
    at = (kv_len - new)[:, None] + i
    sees = there[:, None, :] & (pos[:, None, :] <= at[:, :, None])
    if W:
        sees = sees & ((pos[:, None, :] > at[:, :, None] - W) | (pos[:, None, :] < S))
    scores = torch.matmul(q * hd ** -0.5, k.transpose(2, 3)).view(n, Hkv, M, rep, C)
    scores.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    scores -= scores.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = scores.exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, Hkv, M * rep, C), v).view(n, Hkv, M, rep, hd) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 2, 1, 3, 4).reshape(n, M, -1).to(pool.dtype)
    live = i < new[:, None]
    st["out"][row[live]] = o[live]
    return st["out"]


def _plain_verify(st):
    logits, start, draft, u, T = st["logits"], st["row_start"].long(), st["draft_tokens"].long(), st["u_accept"].double(), st["temperature"]
    rows, V = logits.shape
    n, M = len(T), st["longest"]
    k = start[1:] - start[:-1] - 1
    i = torch.arange(M, device="cuda")
    row = (start[:-1, None] + i).clamp_(max=rows - 1)
    of_row = torch.searchsorted(start[1:], torch.arange(rows, device="cuda"), right=True)
    greedy = T[of_row] <= 0
    index = torch.arange(V, device="cuda")
    best = torch.where(logits == logits.amax(-1, keepdim=True), index, V).amin(-1)
    z = logits.double() / torch.where(greedy, 1.0, T[of_row].double())[:, None]
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p /= p.sum(-1, keepdim=True)
    p = torch.where(greedy[:, None], (index == best[:, None]).double(), p)
    px = p.gather(1, draft[:, None])[:, 0]
    qx = st["draft_probs"].gather(1, draft[:, None])[:, 0].double() if st["draft_probs"] is not None else torch.ones_like(px)
    ok = torch.where(greedy, draft == best, u * qx < px)
    accepted = (ok[row] & (i < k[:, None])).long().cumprod(1).sum(1)
    at = start[:-1] + accepted
    r = p[at]
    q = st["draft_probs"][at].double() if st["draft_probs"] is not None else (index == draft[at][:, None]).double()
    rest = torch.where(((accepted < k) & ~greedy[at])[:, None], (r - q).clamp_(min=0), r)
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, r)
    cum = rest.cumsum(-1)
    hit = (cum > st["u_pick"].double()[:, None] * cum[:, -1:]) & (rest > 0)
    last = torch.where(rest > 0, index, 0).amax(-1)
    token = torch.where(hit, index, V).amin(-1)
    token = torch.where(token < V, token, last)
    tokens = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    j = torch.arange(rows, device="cuda") - start[of_row]
    tokens = torch.where(j < accepted[of_row], draft, torch.where(j == accepted[of_row], token[of_row], -1)).to(torch.int32)
    return {"tokens": tokens, "accepted": accepted.to(torch.int32)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] in ("tables", "verify"):
        return None   # whole numbers
    st = prepare(case, seed)
    s = st["model"]
    Hq, Hkv, hd = s.n_q_heads, s.n_kv_heads, s.head_dim
    if case["op"] == "norm_rope":
        x = st["qkv"].double().view(-1, Hq + 2 * Hkv, hd)
        kv = st["pool"][st["layer"]].double()
        e = torch.arange(hd // 2, device="cuda", dtype=torch.float64) * (-2.0 / hd)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["positions"].double()[:, None] * torch.pow(torch.tensor(s.rope_theta, dtype=torch.float64, device="cuda"), e))
        q = torch.empty(len(x), Hq, hd, dtype=torch.float64, device="cuda")
        block, at = st["slots"].long() // BS, st["slots"].long() % BS
        for h in range(Hq + Hkv):   # a head at a time, pairs as complex numbers
            y, gain = x[:, h], st["q_gain"] if h < Hq else st["k_gain"]
            if gain is not None:
                y = gain.double() * y / (y.norm(dim=-1, keepdim=True) ** 2 / hd + s.rms_eps).sqrt()
            w = torch.complex(y[:, :hd // 2].contiguous(), y[:, hd // 2:].contiguous()) * turn
            y = torch.cat([w.real, w.imag], -1)
            if h < Hq:
                q[:, h] = y
            else:
                kv[0][block, h - Hq, at] = y
        for h in range(Hkv):
            kv[1][block, h, at] = x[:, Hq + Hkv + h]
        return {"q": q.view(len(x), -1), "kv": kv}
    start, kv_len, table = st["row_start"].tolist(), st["kv_len"].tolist(), st["table"].tolist()
    out = torch.zeros(len(st["q"]), Hq, hd, dtype=torch.float64, device="cuda")
    q = st["q"].double().view(-1, Hq, hd)
    for r, end in enumerate(kv_len):   # a request at a time, a few rows at a time
        first = end - (start[r + 1] - start[r])
        for a in range(start[r], start[r + 1], 512):
            b = min(a + 512, start[r + 1])
            p0 = first + a - start[r]
            lo = max(0, p0 - st["window"] + 1) if st["window"] else 0
            pos = torch.tensor(sorted(set(range(min(st["sinks"], p0 + b - a))) | set(range(lo, p0 + b - a))), device="cuda")
            where = torch.tensor(table[r], device="cuda")[pos // BS]
            p = p0 + torch.arange(b - a, device="cuda")[:, None]
            see = pos <= p
            if st["window"]:
                see &= (p - pos < st["window"]) | (pos < st["sinks"])
            for h in range(Hkv):
                kh, vh = (st["pool"][0, i][where, h, pos % BS].double() for i in (0, 1))
                heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
                sc = torch.einsum("thd,cd->htc", q[a:b, heads], kh) / math.sqrt(hd)
                pr = torch.softmax(sc.masked_fill(~see, -math.inf), -1)
                out[a:b, heads] = torch.einsum("htc,cd->thd", pr, vh)
    return out.view(len(out), -1)
