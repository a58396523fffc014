"""Speed of the operators of a paged key/value cache and of the attention that reads it, with seeded inputs.

A case is one call (or, for `turnover`, the calls that follow one another) on a cache of 16-token blocks:
  decode    axon_attn_decode: one query per row over its cached tokens, with an optional sliding window and sinks;
  prompt    axon_attn_prefill: chunks of new tokens after their rows' cached ones, packed row after row;
  fork      axon_kv_fork: rows that take over other rows' blocks, the part-filled last one copied;
  compact   axon_kv_compact: the blocks in use moved to the front of the pool, tables and counts rewritten;
  turnover  axon_kv_release of rows that end, and of what others slid past, then axon_kv_reserve of what these need next.

Lengths go by the case alone, spread evenly over its range; the seed draws values, the order of lengths and the blocks' places.
Calls that change tables and counts begin with putting back the ones that the state started from: one copy on either side.
With `own` false the operators run in their plain form: whole-tensor operations of torch in 32 bits, rounded once.
"""
import math

import numpy as np
import torch

own = False

BS = 16  # tokens per block
# attention shapes of the benchmarked decoders: query heads, kv heads, head_dim, layers
HEADS = {"135m": (9, 3, 64, 30), "0.5b": (14, 2, 64, 24), "8b": (32, 8, 128, 32), "32b": (40, 8, 128, 64),
         "moe16b": (16, 16, 128, 28), "7b_swa": (32, 8, 128, 32)}


def listed():
    return [
        # single-stream generation of a small model: latency
        dict(name="decode_b1", op="decode", model="0.5b", prec="bf16", B=1, lo=577, hi=577, window=0, sinks=0),
        # a server's batch of ragged streams, the long ones past their window
        dict(name="decode_b64_sinks", op="decode", model="8b", prec="fp16", B=64, lo=512, hi=4096, window=2048, sinks=4),
        # one stream with a very long context: the keys have to be spread over the GPU
        dict(name="decode_long", op="decode", model="8b", prec="bf16", B=1, lo=131071, hi=131071, window=0, sinks=0),
        # a short prompt of the smallest model: latency
        dict(name="prompt_s16", op="prompt", model="135m", prec="bf16", B=1, new_lo=16, new_hi=16, past_lo=0, past_hi=0,
             ones=0, window=0, sinks=0),
        # a pass of a continuously batching server: single tokens and pieces of prompts, under a window with sinks
        dict(name="prompt_mixed", op="prompt", model="8b", prec="bf16", B=3, new_lo=257, new_hi=777, past_lo=64, past_hi=900,
             ones=21, window=512, sinks=4),
        # a long prompt under a window with sinks
        dict(name="prompt_s8191_sinks", op="prompt", model="7b_swa", prec="fp16", B=1, new_lo=8191, new_hi=8191, past_lo=0,
             past_hi=0, ones=0, window=4096, sinks=4),
        # four samples from one prompt, small model
        dict(name="fork_samples", op="fork", model="0.5b", prec="bf16", layers=24, groups=1, width=4, lo=577, hi=577,
             beam=False),
        # a step of beam search, 16 prompts of 4 beams, half of the layers
        dict(name="fork_beams", op="fork", model="8b", prec="fp16", layers=16, groups=16, width=4, lo=512, hi=4096, beam=True),
        # a small server's pool after many short requests
        dict(name="compact_small", op="compact", model="0.5b", prec="bf16", layers=24, blocks=509, share=40, rows=16),
        # a large pool at half its fill
        dict(name="compact_large", op="compact", model="8b", prec="fp16", layers=8, blocks=6000, share=50, rows=64),
        # one serving step of a few streams: blocks slide out, new ones are taken
        dict(name="turnover_b8", op="turnover", rows=8, lo=577, hi=2048, ends=1, new=16, window=512, sinks=4, spare=64),
        # a large server's step with chunks of prompts: many rows, a large pool
        dict(name="turnover_b512", op="turnover", rows=512, lo=512, hi=4096, ends=64, new=300, window=1024, sinks=4,
             spare=20000),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["decode", "decode", "prompt", "prompt", "fork", "compact", "turnover"])
    model = rng.choice(sorted(HEADS))
    c = dict(op=op, model=model, prec=rng.choice(["bf16", "fp16"]))
    G, d, L = HEADS[model][1:]
    windowed = rng.random() < 0.6
    if op == "decode":
        c["B"] = log_int(1, 64)
        # as many bytes of keys and values as the largest listed case at most
        hi = log_int(1, max(1, min(131071, 131071 * 8 * 128 // (G * d * c["B"]))))
        c.update(lo=rng.randint(max(1, hi // 4), hi), hi=hi)
        c.update(window=log_int(1, 8192) if windowed else 0)
        c.update(sinks=rng.choice([0, 1, 4, 16, 33]) if windowed else 0)
    elif op == "prompt":
        rows = log_int(1, 3000)
        c["B"] = log_int(1, min(8, rows))
        hi = max(1, rows // c["B"])
        past = log_int(1, 2000) if rng.random() < 0.5 else 0
        c.update(new_lo=rng.randint(max(1, hi // 3), hi), new_hi=hi, past_lo=past // 2, past_hi=past,
                 ones=log_int(1, 16) if rng.random() < 0.3 else 0)
        c.update(window=log_int(1, 2048) if windowed else 0)
        c.update(sinks=rng.choice([0, 1, 4, 16, 33]) if windowed else 0)
    elif op == "fork":
        c.update(layers=rng.randint(1, 4), groups=log_int(1, 16), width=rng.randint(2, 5), hi=log_int(17, 2000),
                 beam=rng.random() < 0.6)
        c["lo"] = rng.randint(max(1, c["hi"] // 4), c["hi"])
    elif op == "compact":
        c.update(layers=rng.randint(1, 6), blocks=log_int(64, 4000), share=rng.randint(10, 95), rows=log_int(1, 64))
    else:
        c = dict(op=op, rows=log_int(2, 400), hi=log_int(64, 4000), new=log_int(1, 400), window=log_int(16, 2048),
                 sinks=rng.choice([0, 1, 4, 16, 33]), spare=log_int(64, 20000))
        c.update(lo=rng.randint(1, c["hi"]), ends=rng.randint(0, c["rows"] // 2))
        c["spare"] += c["rows"] * (c["new"] // BS + 1)
    return c


# ------------------------------------------------------------------ inputs


def _spread(lo, hi, n):
    """n lengths of lo .. hi, evenly spaced."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _type(case):
    return torch.float16 if case.get("prec") == "fp16" else torch.bfloat16


def _int(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()


def _blocks_of(n):
    return -(-n // BS)


def _sequences(case):
    """(cached before, new) tokens of each row of an attention case, in the order of the case."""
    if case["op"] == "decode":
        return [(n - 1, 1) for n in _spread(case["lo"], case["hi"], case["B"])]
    past = _spread(case["past_lo"], case["past_hi"], case["B"] + case["ones"])
    new = _spread(case["new_lo"], case["new_hi"], case["B"]) + [1] * case["ones"]
    return list(zip(past, new))


def _attn_plan(case, seed):
    r = np.random.Generator(np.random.PCG64(seed + 101))
    seqs = _sequences(case)
    seqs = [seqs[i] for i in r.permutation(len(seqs))]
    need = [_blocks_of(p + n) for p, n in seqs]
    P, N = max(need), sum(need) + 8
    perm = r.permutation(N)
    table = np.full((len(seqs), P), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return seqs, table, N


def _normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return t.mul_(scale) if scale != 1.0 else t


def _pages_plan(case, seed):
    """Block table, lengths and reference counts of a cache in use, and what the call is asked."""
    r = np.random.Generator(np.random.PCG64(seed + 202))
    op = case["op"]
    if op == "fork":
        lens = [n for n in _spread(case["lo"], case["hi"], case["groups"])]
        lens = [lens[i] for i in r.permutation(len(lens))]
        w = case["width"]
        per = w if case["beam"] else 1 + w  # rows of a group
        R = len(lens) * per
        P = _blocks_of(max(lens)) + 2
        holders = w if case["beam"] else 1
        need = sum(_blocks_of(n) + (holders - 1) * (n % BS > 0) for n in lens) + w * len(lens) + 8
        perm, at = r.permutation(need), 0
        table, ctx, refs = np.full((R, P), -1), np.zeros(R, dtype=int), np.zeros(need, dtype=int)
        for g, n in enumerate(lens):
            whole = perm[at:at + n // BS]
            at += len(whole)
            for k in range(holders):
                row = g * per + k
                table[row, :len(whole)] = whole
                refs[whole] += 1
                ctx[row] = n
                if n % BS:
                    table[row, n // BS] = perm[at]
                    refs[perm[at]] = 1
                    at += 1
        if case["beam"]:
            dst = np.arange(R)
            src = dst // w * w + r.integers(0, w, R)
        else:
            dst = np.array([g * per + 1 + k for g in range(len(lens)) for k in range(w)])
            src = dst // per * per
        return table, ctx, refs, dict(src=src, dst=dst)
    if op == "compact":
        N, R = case["blocks"], case["rows"]
        live = max(1, N * case["share"] // 100)
        held = r.permutation(N)[:live]
        refs = np.zeros(N, dtype=int)
        refs[held] = 1
        P = _blocks_of(live * BS // R) + 2
        parts = np.array_split(held, R)
        table, ctx = np.full((R, P), -1), np.zeros(R, dtype=int)
        for b, part in enumerate(parts):
            table[b, :len(part)] = part
            ctx[b] = len(part) * BS
        for b in range(1, R, 2):  # every other row shares its neighbour's first block
            if ctx[b] and ctx[b - 1] and P > len(parts[b]):
                table[b, 1:len(parts[b]) + 1] = parts[b]
                table[b, 0] = parts[b - 1][0]
                refs[parts[b - 1][0]] += 1
                ctx[b] += BS
        return table, ctx, refs, {}
    R = case["rows"]
    lens = _spread(case["lo"], case["hi"], R)
    ctx = np.array([lens[i] for i in r.permutation(R)])
    need = [_blocks_of(n) for n in ctx]
    P = _blocks_of(case["hi"] + case["new"]) + 1
    N = sum(need) + case["spare"]
    perm, at = r.permutation(N), 0
    table, refs = np.full((R, P), -1), np.zeros(N, dtype=int)
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        refs[perm[at:at + n]] = 1
        at += n
    rows = r.permutation(R)
    return table, ctx, refs, dict(ends=rows[:case["ends"]], stays=rows[case["ends"]:],
                                  new=r.integers(1, case["new"] + 1, R - case["ends"]))


class _State:
    plan = None  # descriptors and workspace that a program makes once, with the first call


def prepare(case, seed):
    st = _State()
    st.case = case
    if case["op"] in ("decode", "prompt"):
        H, G, d, _ = HEADS[case["model"]]
        seqs, table, N = _attn_plan(case, seed)
        rows = sum(n for _, n in seqs)
        st.k, st.v = (_normal((1, N, G, BS, d), _type(case), seed * 10 + i) for i in (1, 2))
        # scores of standard deviation 1.6, as a decoder's have
        st.q = _normal((rows, H, d), _type(case), seed * 10 + 3, 1.6)
        st.table = _int(table)
        st.ctx = _int([p for p, _ in seqs])
        st.cu = _int(np.concatenate([[0], np.cumsum([n for _, n in seqs])]))
        st.longest = max(n for _, n in seqs)
        st.o = torch.empty_like(st.q)
        st.lse = torch.empty(rows, H, dtype=torch.float32, device="cuda")
        return st
    table, ctx, refs, asked = _pages_plan(case, seed)
    if case["op"] == "turnover":
        G, d, L = 1, 64, 1  # no block's contents are touched
    else:
        (_, G, d, _), L = HEADS[case["model"]], case["layers"]
    st.k, st.v = (_normal((L, len(refs), G, BS, d), _type(case), seed * 10 + i) for i in (1, 2))
    st.start = _int(np.concatenate([table.reshape(-1), ctx, refs]))
    st.now = st.start.clone()
    R, P = table.shape
    st.table, st.ctx, st.refs = st.now[:R * P].view(R, P), st.now[R * P:R * P + R], st.now[R * P + R:]
    for k, v in asked.items():
        setattr(st, k, _int(v))
    if case["op"] == "compact":
        st.map = torch.empty(len(refs), dtype=torch.int32, device="cuda")
        st.live = torch.empty(1, dtype=torch.int32, device="cuda")
    return st


def run(st):
    c = st.case
    op = c["op"]
    if op in ("decode", "prompt"):
        if own:
            import paper_2608_19889_gb300 as ax
            if st.plan is None:
                cache = ax.make_kv_cache(st.k, st.v)
                st.plan = cache, None if op == "prompt" else ax.make_attn_workspace(cache, st.q.shape[0], st.q.shape[1])
            cache, work = st.plan
            if op == "decode":
                ax.axon_attn_decode(cache, 0, st.q, st.ctx, st.o, work, block_table=st.table, window=c["window"],
                                    sinks=c["sinks"], lse=st.lse)
            else:
                ax.axon_attn_prefill(cache, 0, st.q, st.cu, st.ctx, st.longest, st.o, block_table=st.table,
                                     window=c["window"], sinks=c["sinks"])
        elif op == "decode":
            _plain_decode(st, c["window"], c["sinks"])
        else:
            _plain_prompt(st, c["window"], c["sinks"])
        return {"o": st.o, "lse": st.lse} if op == "decode" else {"o": st.o}
    st.now.copy_(st.start)
    if own:
        import paper_2608_19889_gb300 as ax
        if st.plan is None:
            cache, seqs = ax.make_kv_cache(st.k, st.v), ax.make_kv_seqs(st.table, st.ctx, st.refs)
            st.plan = cache, seqs, ax.make_kv_workspace(cache, seqs)
        cache, seqs, work = st.plan
        if op == "fork":
            ax.axon_kv_fork(cache, seqs, st.src, st.dst, work)
        elif op == "compact":
            ax.axon_kv_compact(cache, seqs, work, moved=st.map, live=st.live)
        else:
            ax.axon_kv_release(cache, seqs, st.ends)
            ax.axon_kv_release(cache, seqs, st.stays, window=c["window"], sinks=c["sinks"])
            ax.axon_kv_reserve(cache, seqs, st.stays, st.new, work)
    elif op == "fork":
        _plain_fork(st)
    elif op == "compact":
        _plain_compact(st)
    else:
        _plain_turnover(st, c["window"], c["sinks"])
    out = {"table": st.table, "ctx": st.ctx, "refs": st.refs}
    if op != "turnover":
        out.update(k=st.k.view(torch.int16), v=st.v.view(torch.int16))  # copies: bit for bit
    if op == "compact":
        out.update(map=st.map, live=st.live)
    return out


# ------------------------------------------------------------------ plain forms


def _gathered(pool, table):
    """[rows, tokens, G, d] in 32 bits."""
    R, P = table.shape
    G, d = pool.shape[2], pool.shape[4]
    return pool[0][table.long().clamp(min=0)].transpose(2, 3).reshape(R, P * BS, G, d).float()


def _visible(pos, tokens, window, sinks):
    """Which of `tokens` keys the queries at `pos` [...] see: [..., tokens]."""
    t = torch.arange(tokens, device="cuda")
    seen = t <= pos[..., None]
    if window:
        seen = seen & ((t > pos[..., None] - window) | (t < sinks))
    return seen


def _attended(q, k, v, seen):
    """q [R, n, H, d], k and v [R, t, G, d], seen [R, n, t] -> outputs and log-sum-exp [R, n, H, ...]; rows that see nothing: 0, -inf."""
    R, n, H, d = q.shape
    G = k.shape[2]
    q = q.float().view(R, n, G, H // G, d).permute(0, 2, 3, 1, 4).reshape(R, G, H // G * n, d)
    s = (q @ k.permute(0, 2, 3, 1)).div_(math.sqrt(d))
    s = s.view(R, G, H // G, n, -1).masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = p.view(R, G, H // G * n, -1) @ v.transpose(1, 2)
    o = o.view(R, G, H // G, n, d) / torch.where(total > 0, total, 1.0)
    lse = (m + total.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(R, n, H, d), lse.permute(0, 3, 1, 2).reshape(R, n, H)


def _plain_decode(st, window, sinks):
    k, v = _gathered(st.k, st.table), _gathered(st.v, st.table)
    seen = _visible(st.ctx, k.shape[1], window, sinks)
    v.masked_fill_(~seen[:, :, None, None], 0.0)
    o, lse = _attended(st.q[:, None], k, v, seen[:, None])
    st.o.copy_(o[:, 0])
    st.lse.copy_(lse[:, 0])


def _plain_prompt(st, window, sinks):
    T, H, d = st.q.shape
    k, v = _gathered(st.k, st.table), _gathered(st.v, st.table)
    row = torch.arange(T, device="cuda")
    b = torch.searchsorted(st.cu[1:].long(), row, right=True)
    i = row - st.cu.long()[b]
    q = torch.zeros(len(st.ctx), st.longest, H, d, dtype=st.q.dtype, device="cuda")
    q[b, i] = st.q
    pos = st.ctx[:, None] + torch.arange(st.longest, device="cuda")
    last = st.ctx + st.cu[1:] - st.cu[:-1]
    v.masked_fill_((torch.arange(v.shape[1], device="cuda") >= last[:, None])[:, :, None, None], 0.0)
    o, _ = _attended(q, k, v, _visible(pos, k.shape[1], window, sinks))
    st.o.copy_(o[b, i])


def _counted(refs, table, sign):
    """refs with `sign` added for every entry of `table` that names a block."""
    flat = table.reshape(-1).long()
    n = refs.shape[0]
    more = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    more.index_add_(0, torch.where(flat >= 0, flat, n), torch.full_like(flat, sign, dtype=torch.int32))
    return refs + more[:n]


def _by_rank(chosen, size):
    """Places of the true values of `chosen`, in order, padded to `size` with -1."""
    rank = torch.where(chosen, chosen.cumsum(0) - 1, size).clamp(max=size)
    out = torch.full((size + 1,), -1, dtype=torch.long, device="cuda")
    out[rank] = torch.arange(len(chosen), device="cuda")
    return out[:size]


def _plain_fork(st):
    src, dst = st.src.long(), st.dst.long()
    P = st.table.shape[1]
    n = st.ctx[src].long()
    j = torch.arange(P, device="cuda")
    same = src == dst
    taken = st.table[src]
    taken = torch.where((j < ((n + BS - 1) // BS)[:, None]) | same[:, None], taken, -1)
    copies = (n % BS > 0) & ~same
    last = (n // BS).clamp(max=P - 1)
    part = st.table[src, last].long()
    shared = torch.where(copies[:, None] & (j == last[:, None]), -1, taken)
    refs = _counted(_counted(st.refs, st.table[dst], -1), shared, 1)
    held = _counted(refs, torch.where(copies, part, -1), 1)
    free = _by_rank(held == 0, len(src))
    mine = free[(copies.cumsum(0) - 1).clamp(min=0)]
    # rows that copy nothing write one of their own blocks onto itself
    come = torch.where(copies, part, st.table[src, 0].long())
    to = torch.where(copies, mine, come)
    st.k[:, to] = st.k[:, come]
    st.v[:, to] = st.v[:, come]
    st.table[dst] = torch.where(copies[:, None] & (j == last[:, None]), mine[:, None].int(), shared)
    st.ctx[dst] = n.int()
    st.refs.copy_(_counted(refs, torch.where(copies, mine, -1), 1))


def _plain_compact(st):
    N = st.refs.shape[0]
    at = torch.arange(N, device="cuda")
    used = st.refs > 0
    live = used.sum()
    holes, high = ~used & (at < live), used & (at >= live)
    hole, source = _by_rank(holes, N), _by_rank(high, N)
    where = torch.where(high, hole[(high.cumsum(0) - 1).clamp(min=0)], at)
    come = torch.where(holes, source[(holes.cumsum(0) - 1).clamp(min=0)], at)
    st.map.copy_(torch.where(used, where, -1))
    st.live.copy_(live)
    st.k.copy_(st.k[:, come])
    st.v.copy_(st.v[:, come])
    st.table.copy_(torch.where(st.table >= 0, st.map[st.table.long().clamp(min=0)], -1))
    st.refs.copy_(torch.where(at < live, st.refs[come], 0))


def _plain_turnover(st, window, sinks):
    ends, stays = st.ends.long(), st.stays.long()
    P = st.table.shape[1]
    j = torch.arange(P, device="cuda")
    refs = _counted(st.refs, st.table[ends], -1)
    st.table[ends] = -1
    st.ctx[ends] = 0
    n = st.ctx[stays].long()
    gone = (j >= -(-sinks // BS)) & ((j + 1) * BS <= (n - window + 1)[:, None])
    rows = st.table[stays]
    refs = _counted(refs, torch.where(gone, rows, -1), -1)
    rows = torch.where(gone, -1, rows)
    wanted = (j >= ((n + BS - 1) // BS)[:, None]) & (j < ((n + st.new + BS - 1) // BS)[:, None]) & (rows < 0)
    flat = wanted.reshape(-1)
    free = _by_rank(refs == 0, flat.numel())
    mine = torch.where(flat, free[(flat.cumsum(0) - 1).clamp(min=0)], -1).view(rows.shape).int()
    st.table[stays] = torch.where(wanted, mine, rows)
    st.refs.copy_(_counted(refs, mine, 1))


# ------------------------------------------------------------------ what a pass cannot do without


def _seen_by(p, window, sinks):
    """Keys that a query at position p sees."""
    return p + 1 if not window or p < window else window + min(sinks, p + 1 - window)


def work(case):
    op = case["op"]
    if op in ("decode", "prompt"):
        H, G, d, _ = HEADS[case["model"]]
        W, s = case["window"], case["sinks"]
        keys = pairs = rows = entries = 0
        for past, new in _sequences(case):
            first = max(0, past + 1 - W) if W else 0  # the first row's window
            keys += past + new - first + min(s, first)
            entries += _blocks_of(past + new) - first // BS
            pairs += sum(_seen_by(past + i, W, s) for i in range(new))
            rows += new
        nbytes = keys * G * d * 2 * 2 + rows * H * d * 2 * 2 + entries * 4
        return {"bytes": nbytes + (rows * H * 4 if op == "decode" else 0), "flops": 4.0 * H * d * pairs}
    if op == "turnover":
        table, _, refs, _ = _pages_plan(case, 1)
        return {"bytes": 4.0 * (2 * int((table >= 0).sum()) + len(refs)), "flops": 0.0}
    _, G, d, _ = HEADS[case["model"]]
    block = case["layers"] * 2 * G * BS * d * 2
    if op == "fork":
        lens = _spread(case["lo"], case["hi"], case["groups"])
        w = case["width"]
        share = (w - 1) / w if case["beam"] else 1.0  # of a group's rows that take another row's place
        moves = sum(n % BS > 0 for n in lens) * w * share
        return {"bytes": 2.0 * block * moves + 8.0 * w * share * sum(_blocks_of(n) for n in lens), "flops": 0.0}
    N = case["blocks"]
    live = max(1, N * case["share"] // 100)
    return {"bytes": 2.0 * block * live * (N - live) / N + 4.0 * (2 * N + 2 * live), "flops": 0.0}


# ------------------------------------------------------------------ the same in 64 bits


def exact(case, seed):
    if case["op"] not in ("decode", "prompt"):
        return None  # whole numbers and copied bits
    H, G, d, _ = HEADS[case["model"]]
    W, sinks = case["window"], case["sinks"]
    seqs, table, N = _attn_plan(case, seed)
    if 8.0 * d * H * sum(n * (p + n) for p, n in seqs) > 1.5e13:
        return None
    k, v = (_normal((1, N, G, BS, d), _type(case), seed * 10 + i)[0] for i in (1, 2))
    q = _normal((sum(n for _, n in seqs), H, d), _type(case), seed * 10 + 3, 1.6)
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    row = 0
    for b, (past, new) in enumerate(seqs):
        total = past + new
        t = torch.arange(total, device="cuda")
        place, inside = torch.from_numpy(table[b]).cuda().long()[t // BS], t % BS
        for at in range(0, new, 1024):
            rows = slice(row + at, row + min(at + 1024, new))
            p = (past + torch.arange(at, min(at + 1024, new), device="cuda"))[:, None]
            hidden = t > p
            if W:
                hidden = hidden | ((t <= p - W) & (t >= sinks))
            for h in range(H):
                g = h // (H // G)
                s = q[rows, h].double() @ k[place, g, inside].double().T / math.sqrt(d)
                s[hidden] = -math.inf
                lse[rows, h] = torch.logsumexp(s, -1)
                o[rows, h] = torch.softmax(s, -1) @ v[place, g, inside].double()
        row += new
    return {"o": o, "lse": lse} if case["op"] == "decode" else {"o": o}
