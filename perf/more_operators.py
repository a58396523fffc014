"""Speed of the operators of a decode step that samples several continuations of one prompt, with seeded inputs.

A case is one call on a cache of 16-token blocks, or on a step's logits:
  append    axon_kv_append: queries and keys of new tokens rotated to their positions, keys and values written to the cache;
  shared    axon_attn_shared: one query per row over its cached tokens, rows in groups whose first blocks are the same;
  sample    axon_sample: a token per row from its logits, by temperature, top-k, top-p, min-p and a given random number.

Sizes and lengths go by the case alone, spread evenly over its range; the seed draws values, orders and the blocks' places.
With `own` false the operators run in their plain form: torch operations in 32 bits, rounded once; sampling, where a
token hangs on which side of a border a sum falls, in 64.
"""
import math

import numpy as np
import torch

own = False

BS = 16  # tokens per block
# attention shapes and vocabularies of the benchmarked decoders: query heads, kv heads, head_dim, vocabulary, rotary base
MODELS = {"135m": (9, 3, 64, 49152, 1e4), "0.5b": (14, 2, 64, 151936, 1e6), "8b": (32, 8, 128, 128256, 5e5),
          "32b": (40, 8, 128, 152064, 1e6), "moe16b": (16, 16, 128, 102400, 1e4), "7b_swa": (32, 8, 128, 32000, 1e4)}
# the frequency scaling of a decoder with a long context: factor, low, high, original positions
SCALING = (8.0, 1.0, 4.0, 8192)


def listed():
    return [
        # a step of single-stream generation of a small model: latency
        dict(name="append_b1", op="append", model="0.5b", prec="bf16", B=1, new_lo=1, new_hi=1, past_lo=577, past_hi=577,
             ones=0, rotary=64, layout="half", scaled=False),
        # a step of a server's batch of ragged streams, positions of a long context
        dict(name="append_b64", op="append", model="8b", prec="fp16", B=64, new_lo=1, new_hi=1, past_lo=512, past_hi=65535,
             ones=0, rotary=128, layout="half", scaled=True),
        # a pass of a continuously batching server: single tokens and pieces of prompts; half of each head is rotated
        dict(name="append_mixed", op="append", model="moe16b", prec="bf16", B=3, new_lo=257, new_hi=777, past_lo=64,
             past_hi=900, ones=21, rotary=64, layout="interleaved", scaled=False),
        # a long prompt
        dict(name="append_s8191", op="append", model="8b", prec="bf16", B=1, new_lo=8191, new_hi=8191, past_lo=0, past_hi=0,
             ones=0, rotary=128, layout="half", scaled=True),
        # four samples from one prompt, small model: latency
        dict(name="shared_samples", op="shared", model="0.5b", prec="bf16", groups=1, width=4, pre_lo=577, pre_hi=577,
             own_lo=1, own_hi=64, alone=0, window=0, sinks=0),
        # a step of beam search, 16 prompts of 4 beams
        dict(name="shared_beams", op="shared", model="8b", prec="fp16", groups=16, width=4, pre_lo=512, pre_hi=4096,
             own_lo=3, own_hi=129, alone=0, window=0, sinks=0),
        # requests with one system prompt, and some without, under a window with sinks
        dict(name="shared_system", op="shared", model="7b_swa", prec="bf16", groups=1, width=48, pre_lo=4001, pre_hi=4001,
             own_lo=1, own_hi=1500, alone=9, window=4096, sinks=4),
        # many questions to one long document
        dict(name="shared_document", op="shared", model="32b", prec="bf16", groups=1, width=64, pre_lo=32768, pre_hi=32768,
             own_lo=16, own_hi=300, alone=0, window=0, sinks=0),
        # one stream: latency
        dict(name="sample_b1", op="sample", model="0.5b", prec="fp32", B=1, shape="peaked", temp_lo=0.7, temp_hi=0.7,
             top_k=50, top_p=0.9, min_p=0.0, mixed=False, masked=False),
        # a batch whose rows all ask for something else, greedy ones among them
        dict(name="sample_mixed", op="sample", model="32b", prec="bf16", B=33, shape="peaked", temp_lo=0.3, temp_hi=1.5,
             top_k=40, top_p=0.95, min_p=0.05, mixed=True, masked=True),
        # samples by top-p alone, a wide distribution: tens of thousands of tokens stay
        dict(name="sample_b64_top_p", op="sample", model="8b", prec="fp32", B=64, shape="flat", temp_lo=1.0, temp_hi=1.0,
             top_k=0, top_p=0.95, min_p=0.0, mixed=False, masked=False),
        # many samples by temperature alone
        dict(name="sample_b512", op="sample", model="7b_swa", prec="fp32", B=512, shape="peaked", temp_lo=0.5, temp_hi=1.2,
             top_k=0, top_p=1.0, min_p=0.0, mixed=False, masked=False),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "append", "shared", "shared", "shared", "sample", "sample", "sample"])
    model = rng.choice(sorted(MODELS))
    H, G, d, V, _ = MODELS[model]
    c = dict(op=op, model=model, prec=rng.choice(["bf16", "fp16"]))
    if op == "append":
        rows = log_int(1, 5000)
        c["B"] = log_int(1, min(64, rows))
        hi = max(1, rows // c["B"])
        past = log_int(1, 30000) if rng.random() < 0.7 else 0
        c.update(new_lo=rng.randint(max(1, hi // 3), hi), new_hi=hi, past_lo=past // 2, past_hi=past,
                 ones=log_int(1, 16) if rng.random() < 0.3 else 0)
        c.update(rotary=rng.choice([32, d // 2, d, d]), layout=rng.choice(["half", "half", "interleaved"]),
                 scaled=rng.random() < 0.4)
    elif op == "shared":
        windowed = rng.random() < 0.3
        rows = log_int(2, 96)
        c["width"] = min(rows, log_int(2, 64))
        c["groups"] = max(1, rows // c["width"])
        c["alone"] = log_int(1, 12) if rng.random() < 0.3 else 0
        # as many bytes of keys, counted for each row, as the largest listed case at most
        most = 2_000_000 * 1024 // (c["groups"] * c["width"] * G * d)
        c["pre_hi"] = log_int(16, max(17, min(40000, most)))
        c["pre_lo"] = rng.randint(max(1, c["pre_hi"] // 4), c["pre_hi"])
        c["own_hi"] = log_int(1, 700)
        c["own_lo"] = rng.randint(1, c["own_hi"])
        c.update(window=log_int(16, 8192) if windowed else 0, sinks=rng.choice([0, 1, 4, 33]) if windowed else 0)
    else:
        c["prec"] = rng.choice(["fp32", "fp32", "fp32", "bf16", "fp16"])
        c["B"] = log_int(1, max(2, min(400, 12_000_000 // V)))
        c.update(shape=rng.choice(["peaked", "peaked", "flat"]), temp_lo=round(rng.uniform(0.1, 1.0), 3),
                 temp_hi=round(rng.uniform(1.0, 2.0), 3), top_k=rng.choice([0, 0, 1, log_int(2, 2000)]),
                 top_p=rng.choice([1.0, round(rng.uniform(0.05, 0.999), 3)]),
                 min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.3), 3)]), mixed=rng.random() < 0.4,
                 masked=rng.random() < 0.3)
    return c


# ------------------------------------------------------------------ inputs


def _spread(lo, hi, n):
    """n lengths of lo .. hi, evenly spaced."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _type(case):
    return {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}[case["prec"]]


def _int(v):
    return torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()


def _blocks_of(n):
    return -(-n // BS)


def _normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
    return t.mul_(scale) if scale != 1.0 else t


def _frequencies(case):
    """Angle per position of each rotated pair, in 64 bits."""
    theta, r = MODELS[case["model"]][4], case["rotary"]
    f = theta ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if case["scaled"]:
        factor, low, high, original = SCALING
        t = np.clip((original * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        f = (1.0 - t) * f / factor + t * f
    return f


def _append_plan(case, seed):
    """(cached before, new) tokens of the rows, a table of the blocks that the new tokens go to, and how many there are."""
    r = np.random.Generator(np.random.PCG64(seed + 301))
    n = case["B"] + case["ones"]
    new = _spread(case["new_lo"], case["new_hi"], case["B"]) + [1] * case["ones"]
    seqs = list(zip(_spread(case["past_lo"], case["past_hi"], n), new))
    seqs = [seqs[i] for i in r.permutation(n)]
    touched = [range(p // BS, _blocks_of(p + m)) for p, m in seqs]
    N = sum(len(t) for t in touched) + 3
    table = np.full((n, max(t.stop for t in touched)), -1, dtype=np.int32)
    perm, at = r.permutation(N), 0
    for b, t in enumerate(touched):
        table[b, t.start:t.stop] = perm[at:at + len(t)]
        at += len(t)
    return seqs, table, N


def _groups(case):
    """Groups of an attention case: (tokens of the shared prefix, lengths of its rows)."""
    out, w = [], case["width"]
    own = _spread(case["own_lo"], case["own_hi"], case["groups"] * w)
    for g, p in enumerate(_spread(case["pre_lo"], case["pre_hi"], case["groups"])):
        out.append((p, [p + n for n in own[g::case["groups"]]]))
    for n in _spread(case["own_hi"], case["pre_hi"] + case["own_hi"], case["alone"]) if case["alone"] else []:
        out.append((0, [n]))
    return out


def _shared_plan(case, seed):
    """Lengths, table, offsets of the groups' rows and their prefixes; blocks that a window hides from all are -1."""
    r = np.random.Generator(np.random.PCG64(seed + 402))
    groups = _groups(case)
    groups = [groups[i] for i in r.permutation(len(groups))]
    groups = [(p, [lens[i] for i in r.permutation(len(lens))]) for p, lens in groups]
    N = sum(p // BS + sum(_blocks_of(n) - p // BS for n in lens) for p, lens in groups) + 5
    rows = sum(len(lens) for _, lens in groups)
    table = np.full((rows, max(_blocks_of(n) for _, lens in groups for n in lens)), -1, dtype=np.int32)
    perm, at, row = r.permutation(N), 0, 0
    for p, lens in groups:
        same = perm[at:at + p // BS]
        at += len(same)
        for n in lens:
            mine = _blocks_of(n) - len(same)
            table[row, :len(same)] = same
            table[row, len(same):len(same) + mine] = perm[at:at + mine]
            at += mine
            row += 1
    lens = np.array([n for _, lens in groups for n in lens])
    offsets = np.concatenate([[0], np.cumsum([len(lens) for _, lens in groups])])
    return lens, table, offsets, np.array([p for p, _ in groups]), N


def _sample_inputs(case, seed):
    """Logits and what each row asks for: temperature (0: the largest logit), top-k (0: all), top-p, min-p, random number."""
    B, V = case["B"], MODELS[case["model"]][3]
    # a wide spread as a random-init decoder has, or a body of unlikely tokens with some likely ones
    x = _normal((B, V), torch.float32, seed * 10 + 5, 1.3 if case["shape"] == "flat" else 2.0)
    r = np.random.Generator(np.random.PCG64(seed + 503))
    if case["shape"] == "peaked":
        part = V // 60  # one likely token in each sixtieth of the vocabulary
        at = torch.from_numpy(r.integers(0, part, (B, 60)) + np.arange(60) * part).cuda()
        x.scatter_(1, at, torch.from_numpy(6.0 + 8.0 * r.random((B, 60)) ** 2).float().cuda())
    if case["masked"]:  # a grammar leaves every third token
        x[:, torch.arange(V, device="cuda") % 3 != int(r.integers(0, 3))] = -math.inf
    temp = np.array(_spread(0, 1000, B)) / 1000.0 * (case["temp_hi"] - case["temp_lo"]) + case["temp_lo"]
    k, p, m = np.full(B, case["top_k"]), np.full(B, case["top_p"]), np.full(B, case["min_p"])
    if case["mixed"]:
        kind = np.arange(B) % 6  # greedy, temperature alone, one of the three, all
        temp[kind == 0] = 0.0
        k[(kind != 2) & (kind != 5)] = 0
        p[(kind != 3) & (kind != 5)] = 1.0
        m[(kind != 4) & (kind != 5)] = 0.0
    u = r.random(B, dtype=np.float32)
    order = r.permutation(B)
    f32 = lambda v: v[order].astype(np.float32)  # noqa: E731
    return x.to(_type(case)), f32(temp), k[order].astype(np.int32), f32(p), f32(m), u


class _State:
    plan = None  # descriptor and workspace that a program makes once, with the first call


def prepare(case, seed):
    st = _State()
    st.case = case
    H, G, d, V, _ = MODELS[case["model"]]
    t = _type(case)
    if case["op"] == "append":
        seqs, table, N = _append_plan(case, seed)
        rows = sum(n for _, n in seqs)
        # the projection's output: queries, keys and values of a token side by side
        qkv = _normal((rows, H + 2 * G, d), t, seed * 10 + 3)
        st.q, st.new_k, st.new_v = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
        st.k, st.v = (_normal((1, N, G, BS, d), t, seed * 10 + i) for i in (1, 2))
        st.table = _int(table)
        st.ctx = _int([p for p, _ in seqs])
        st.cu = _int(np.concatenate([[0], np.cumsum([n for _, n in seqs])])) if rows > len(seqs) else None
        angle = torch.arange(max(p + n for p, n in seqs), dtype=torch.float64, device="cuda")[:, None] * \
            torch.from_numpy(_frequencies(case)).cuda()
        st.rope = torch.stack([angle.cos(), angle.sin()], -1).float()
        st.o = torch.empty(rows, H, d, dtype=t, device="cuda")
    elif case["op"] == "shared":
        lens, table, offsets, prefixes, N = _shared_plan(case, seed)
        st.k, st.v = (_normal((1, N, G, BS, d), t, seed * 10 + i) for i in (1, 2))
        # scores of standard deviation 1.6, as a decoder's have
        st.q = _normal((len(lens), H, d), t, seed * 10 + 3, 1.6)
        st.table, st.ctx, st.offsets, st.prefixes = _int(table), _int(lens - 1), _int(offsets), _int(prefixes)
        st.o = torch.empty_like(st.q)
        st.lse = torch.empty(len(lens), H, dtype=torch.float32, device="cuda")
    else:
        st.x, *asked = _sample_inputs(case, seed)
        st.temp, st.top_k, st.top_p, st.min_p, st.u = (torch.from_numpy(a).cuda() for a in asked)
        st.token = torch.empty(case["B"], dtype=torch.int32, device="cuda")
        st.prob = torch.empty(case["B"], dtype=torch.float32, device="cuda")
    return st


def run(st):
    c = st.case
    if c["op"] == "append":
        if own:
            import paper_2608_19889_gb300 as ax
            if st.plan is None:
                st.plan = ax.make_kv_cache(st.k, st.v)
            ax.axon_kv_append(st.plan, 0, st.new_k, st.new_v, st.ctx, block_table=st.table, cu_seqlens=st.cu, rope=st.rope,
                              interleaved=c["layout"] == "interleaved", q=st.q, q_out=st.o)
        else:
            _plain_append(st)
        return {"q": st.o, "k": st.k, "v": st.v}
    if c["op"] == "shared":
        if own:
            import paper_2608_19889_gb300 as ax
            if st.plan is None:
                cache = ax.make_kv_cache(st.k, st.v)
                st.plan = cache, ax.make_shared_workspace(cache, st.q.shape[0], st.q.shape[1])
            cache, work = st.plan
            ax.axon_attn_shared(cache, 0, st.q, st.ctx, st.offsets, st.prefixes, st.o, work, st.table, window=c["window"],
                                sinks=c["sinks"], lse=st.lse)
        else:
            _plain_shared(st)
        return {"o": st.o, "lse": st.lse}
    if own:
        import paper_2608_19889_gb300 as ax
        ax.axon_sample(st.x, st.u, st.token, temperature=st.temp, top_k=st.top_k, top_p=st.top_p, min_p=st.min_p,
                       prob=st.prob)
    else:
        _plain_sample(st)
    return {"token": st.token, "prob": st.prob}


# ------------------------------------------------------------------ plain forms


def _turned(x, turn, interleaved):
    """x [rows, heads, d] in 32 bits with its first pairs turned by turn [rows, pairs, 2] (cosine, sine)."""
    n = turn.shape[1]
    c, s = turn[:, None, :, 0], turn[:, None, :, 1]
    out = x.float().clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    xa, xb = x[..., a].float(), x[..., b].float()
    out[..., a] = xa * c - xb * s
    out[..., b] = xb * c + xa * s
    return out


def _plain_append(st):
    rows = st.q.shape[0]
    row = torch.arange(rows, device="cuda")
    if st.cu is None:
        b, pos = row, st.ctx.long()
    else:
        b = torch.searchsorted(st.cu[1:].long(), row, right=True)
        pos = st.ctx.long()[b] + row - st.cu.long()[b]
    turn = st.rope[pos]
    inter = st.case["layout"] == "interleaved"
    st.o.copy_(_turned(st.q, turn, inter))
    block, inside = st.table.long()[b, pos // BS], pos % BS
    at = block[:, None], torch.arange(st.k.shape[2], device="cuda"), inside[:, None]
    st.k[0][at] = _turned(st.new_k, turn, inter).to(st.k.dtype)
    st.v[0][at] = st.new_v


def _plain_shared(st):
    R, H, d = st.q.shape
    G, P = st.k.shape[2], st.table.shape[1]
    W, sinks = st.case["window"], st.case["sinks"]
    t = torch.arange(P * BS, device="cuda")
    step = max(1, (1 << 28) // (P * BS * G * d))  # rows whose keys are gathered at a time
    for at in range(0, R, step):
        rows = slice(at, min(at + step, R))
        pos = st.ctx[rows].long()[:, None]
        seen = t <= pos
        if W:
            seen = seen & ((t > pos - W) | (t < sinks))
        n = seen.shape[0]
        place = st.table[rows].long().clamp(min=0)
        k = st.k[0][place].permute(0, 2, 1, 3, 4).reshape(n, G, P * BS, d).float()
        q = st.q[rows].float().view(n, G, H // G, d)
        s = (q @ k.transpose(2, 3)).div_(math.sqrt(d)).masked_fill_(~seen[:, None, None], -math.inf)
        del k
        m = s.amax(-1, keepdim=True)
        p = s.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        v = st.v[0][place].permute(0, 2, 1, 3, 4).reshape(n, G, P * BS, d).float()
        v.masked_fill_(~seen[:, None, :, None], 0.0)
        st.o[rows] = ((p @ v) / total).view(n, H, d).to(st.o.dtype)
        st.lse[rows] = (m + total.log()).view(n, H)


def _plain_sample(st):
    x, at = torch.sort(st.x.float(), dim=-1, descending=True, stable=True)
    V = x.shape[1]
    greedy = st.temp <= 0
    temp = torch.where(greedy, 1.0, st.temp).double()[:, None]
    w = ((x.double() - x[:, :1].double()) / temp).exp_()
    rank = torch.arange(V, device="cuda")
    k = torch.where(st.top_k > 0, st.top_k, V)[:, None]
    w.masked_fill_(rank >= k, 0.0)
    c = w.cumsum(-1)
    before = torch.cat([torch.zeros_like(c[:, :1]), c[:, :-1]], -1)
    top_p = torch.where(st.top_p < 1, st.top_p, math.inf).double()[:, None]
    kept = (before < top_p * c[:, -1:]) & (w >= st.min_p.double()[:, None]) & ~(greedy[:, None] & (rank > 0))
    kept[:, 0] = True
    w = torch.zeros_like(w).scatter_(1, at, w.masked_fill_(~kept, 0.0))
    c = w.cumsum(-1)
    token = torch.searchsorted(c, st.u.double()[:, None] * c[:, -1:], right=True).clamp(max=V - 1)
    st.token.copy_(token[:, 0])
    st.prob.copy_((w.gather(1, token) / c[:, -1:])[:, 0])


# ------------------------------------------------------------------ what a pass cannot do without


def _keys_seen(first, last, window, sinks):
    """Keys that the query at position `last` sees among those from `first` on."""
    lo = max(0, last + 1 - window) if window else 0
    return max(0, last + 1 - max(first, lo)) + max(0, min(sinks if window else 0, lo) - first)


def work(case):
    H, G, d, V, _ = MODELS[case["model"]]
    if case["op"] == "append":
        n = case["B"] + case["ones"]
        tokens = sum(_spread(case["new_lo"], case["new_hi"], case["B"])) + case["ones"]
        return {"bytes": 4.0 * tokens * (H + 2 * G) * d + 4.0 * tokens * case["rotary"] + 8.0 * n + 4.0 * tokens / BS,
                "flops": 3.0 * tokens * (H + G) * case["rotary"]}
    if case["op"] == "shared":
        W, sinks = case["window"], case["sinks"]
        keys = pairs = rows = 0
        for p, lens in _groups(case):
            p = p // BS * BS
            # of the shared blocks what any row sees, once; of the others what their row sees
            low = min(max(0, n - W) if W else 0 for n in lens)
            keys += max(0, p - low) + min(sinks if W else 0, low, p) + sum(_keys_seen(p, n - 1, W, sinks) for n in lens)
            pairs += sum(_keys_seen(0, n - 1, W, sinks) for n in lens)
            rows += len(lens)
        return {"bytes": 4.0 * keys * G * d + 4.0 * rows * H * d + 4.0 * rows * H + 4.0 * keys / BS,
                "flops": 4.0 * H * d * pairs}
    size = 4 if case["prec"] == "fp32" else 2
    return {"bytes": float(size) * case["B"] * V + 28.0 * case["B"], "flops": 3.0 * case["B"] * V}


# ------------------------------------------------------------------ the same in 64 bits


def exact(case, seed):
    return {"append": _exact_append, "shared": _exact_shared, "sample": _exact_sample}[case["op"]](case, seed)


def _exact_append(case, seed):
    H, G, d, _, _ = MODELS[case["model"]]
    seqs, table, N = _append_plan(case, seed)
    rows = sum(n for _, n in seqs)
    x = _normal((rows, H + 2 * G, d), _type(case), seed * 10 + 3).double()
    k, v = (_normal((1, N, G, BS, d), _type(case), seed * 10 + i).double() for i in (1, 2))
    pos = torch.cat([torch.arange(p, p + n, device="cuda") for p, n in seqs])
    f, r = torch.from_numpy(_frequencies(case)).cuda(), case["rotary"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None, None] * f)
    head = x[:, :H + G]
    if case["layout"] == "interleaved":
        z = torch.view_as_complex(head[..., :r].reshape(rows, H + G, r // 2, 2).contiguous()) * turn
        head[..., :r] = torch.view_as_real(z).reshape(rows, H + G, r)
    else:
        z = torch.complex(head[..., :r // 2], head[..., r // 2:r]) * turn
        head[..., :r] = torch.cat([z.real, z.imag], -1)
    row = 0
    for b, (p, n) in enumerate(seqs):
        at = torch.arange(p, p + n, device="cuda")
        place = torch.from_numpy(table[b]).cuda().long()[at // BS]
        k[0, place, :, at % BS] = x[row:row + n, H:H + G]
        v[0, place, :, at % BS] = x[row:row + n, H + G:]
        row += n
    return {"q": x[:, :H].clone(), "k": k, "v": v}


def _exact_shared(case, seed):
    H, G, d, _, _ = MODELS[case["model"]]
    W, sinks = case["window"], case["sinks"]
    lens, table, _, _, N = _shared_plan(case, seed)
    k, v = (_normal((1, N, G, BS, d), _type(case), seed * 10 + i)[0] for i in (1, 2))
    q = _normal((len(lens), H, d), _type(case), seed * 10 + 3, 1.6).double()
    o, lse = torch.zeros_like(q), torch.zeros_like(q[..., 0])
    for b, n in enumerate(lens.tolist()):
        t = torch.arange(n, device="cuda")
        if W:
            t = t[(t >= n - W) | (t < sinks)]
        place, inside = torch.from_numpy(table[b]).cuda().long()[t // BS], t % BS
        for g in range(G):
            h = slice(g * (H // G), (g + 1) * (H // G))
            s = q[b, h] @ k[place, g, inside].double().T / math.sqrt(d)
            lse[b, h] = torch.logsumexp(s, -1)
            o[b, h] = torch.softmax(s, -1) @ v[place, g, inside].double()
    return {"o": o, "lse": lse}


def _exact_sample(case, seed):
    x, temp, top_k, top_p, min_p, u = _sample_inputs(case, seed)
    x = x.double().cpu().numpy()
    token, prob = np.zeros(len(x), dtype=np.int32), np.ones(len(x))
    for b, row in enumerate(x):
        best = int(row.argmax())
        token[b] = best
        if temp[b] <= 0:
            continue
        w = np.exp((row - row[best]) / np.float64(temp[b]))
        order = np.lexsort((np.arange(len(row)), -row))  # the largest first, of equal ones the lowest number
        if top_k[b] > 0:
            order = order[:top_k[b]]
        if top_p[b] < 1:
            total = np.cumsum(w[order])
            order = order[:1 + int(np.searchsorted(total, np.float64(top_p[b]) * total[-1]))]
        order = np.sort(order[(w[order] >= np.float64(min_p[b])) | (np.arange(len(order)) == 0)])
        total = np.cumsum(w[order])
        i = int(np.searchsorted(total, np.float64(u[b]) * total[-1], side="right"))
        token[b], prob[b] = order[i], w[order[i]] / total[-1]
    return {"token": torch.from_numpy(token), "prob": torch.from_numpy(prob)}
