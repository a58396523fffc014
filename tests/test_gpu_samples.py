"""The operators of a step that draws several samples of one prompt, together: blocks shared by a fork, new tokens appended with
rotation, attention over the shared prefix, tokens drawn; and the same through PagedSeqs and a model.

Attention's tolerance is that of test_gpu_shared.py (5e-4 max |v| and a unit of the output), on keys that the test rotates
itself: they differ from the cache's by the cache's rounding at most half a unit of a key, which is why the reference reads
the cache for keys (append has its own test) and only its own bookkeeping for places."""
import os
import sys

import numpy as np
import pytest

import kv_model as km

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ax():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_19889_gb300 import build
    build.build()
    import paper_2608_19889_gb300 as ax
    return ax


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def drawn(logits, temp, k, p, u):
    """The token that 64-bit arithmetic draws, or None next to a border."""
    row = logits.double().cpu().numpy()
    if temp <= 0:
        return int(row.argmax())
    w = np.exp((row - row.max()) / np.float64(np.float32(temp)))
    order = np.lexsort((np.arange(len(row)), -row))[:k]
    c = np.cumsum(w[order])
    at = np.float64(np.float32(p)) * c[-1]
    near = np.abs(c - at).min() < 1e-9 * c[-1]
    order = np.sort(order[:1 + int(np.searchsorted(c, at))])
    c = np.cumsum(w[order])
    near |= np.abs(c - u * c[-1]).min() < 1e-9 * c[-1]
    return None if near else int(order[int(np.searchsorted(c, u * c[-1], side="right"))])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,G,d", [(8, 2, 64), (32, 8, 128)])
def test_a_step_of_samples(ax, monkeypatch, H, G, d, dtype):
    monkeypatch.setenv("AXON_SHARED_MIN_BYTES", "0")
    r = np.random.default_rng(H)
    rows, per, layers, V = 7, 40, 2, 500
    prompts, widths = [333, 160], [4, 3]  # rows 0..3 and 4..6
    k = torch.full((layers, 120, G, 16, d), float("nan"), dtype=dtype, device=DEV)
    v = torch.full_like(k, float("nan"))
    cache = ax.make_kv_cache(k, v)
    table, lens, refs = torch.full((rows, per), -1, dtype=torch.int32, device=DEV), ints(*[0] * rows), ints(*[0] * 120)
    seqs = ax.make_kv_seqs(table, lens, refs)
    kvw, work, err = ax.make_kv_workspace(cache, seqs), ax.make_shared_workspace(cache, rows, H), ints(0)
    rope = ax.axon_rope_table(per * 16, d, 1e4)
    make = lambda *shape: torch.from_numpy(r.standard_normal(shape)).to(dtype).to(DEV)  # noqa: E731
    # the prompts of rows 0 and 4
    first = ints(0, 4)
    ax.axon_kv_reserve(cache, seqs, first, ints(*prompts), kvw, err=err)
    keys, values = make(sum(prompts), G, d), make(sum(prompts), G, d)
    for layer in range(layers):
        ax.axon_kv_append(cache, layer, keys, values, lens[first.long()].contiguous(), table[first.long()].contiguous(),
                          cu_seqlens=ints(0, prompts[0], sum(prompts)), rope=rope, err=err)
    lens[first.long()] += ints(*prompts)
    ax.axon_kv_fork(cache, seqs, ints(0, 0, 0, 4, 4), ints(1, 2, 3, 5, 6), kvw, err=err)
    offsets, prefix = ints(0, 4, 7), ints(*prompts)
    every, one = torch.arange(rows, dtype=torch.int32, device=DEV), ints(*[1] * rows)
    head = torch.from_numpy(r.standard_normal((H * d, V)) / 4).float().to(DEV)
    temp = torch.tensor([0.0, 0.7, 1.0, 1.3, 0.7, 0.9, 1.1], device=DEV)
    top_k, top_p = ints(*[40] * rows), torch.full((rows,), 0.9, device=DEV)
    tokens, prob = ints(*[0] * rows), torch.empty(rows, device=DEV)
    differ = 0
    for step in range(18):  # past a block's end
        ax.axon_kv_reserve(cache, seqs, every, one, kvw, err=err)
        q, out, lse = make(rows, H, d) * 1.6, torch.empty(rows, H, d, dtype=dtype, device=DEV), torch.empty(rows, H, device=DEV)
        new = make(rows, 2 * G, d)
        for layer in range(layers):
            ax.axon_kv_append(cache, layer, new[:, :G], new[:, G:], lens, table, rope=rope, q=q if layer == layers - 1 else None,
                              q_out=q if layer == layers - 1 else None, err=err)
        ax.axon_attn_shared(cache, layers - 1, q, lens, offsets, prefix, out, work, table, lse=lse, err=err)
        logits = out.float().view(rows, H * d) @ head
        u = torch.from_numpy(r.random(rows, dtype=np.float32)).to(DEV)
        ax.axon_sample(logits, u, tokens, temperature=temp, top_k=top_k, top_p=top_p, prob=prob)
        got, vmax = out.double().cpu().numpy(), float(values.abs().max())
        pool_k, pool_v, at = k[layers - 1].double().cpu().numpy(), v[layers - 1].double().cpu().numpy(), table.cpu().numpy()
        for b, n in enumerate((lens + 1).tolist()):
            assert n == prompts[b >= 4] + step + 1
            places = [(at[b, t // 16], t % 16) for t in range(n)]
            kk, vv = (np.stack([pool[blk, :, i] for blk, i in places]) for pool in (pool_k, pool_v))
            want, _ = km.attention(q[b].double().cpu().numpy(), kk, vv, n - 1, 0, 0)
            off = np.abs(got[b] - want) - torch.finfo(dtype).eps * np.abs(want)
            assert off.max() <= 5e-4 * max(vmax, np.abs(vv).max())
            tok = drawn(logits[b], float(temp[b]), 40, 0.9, float(u[b]))
            assert tok is None or tokens[b].item() == tok
        differ += len(set(tokens.tolist())) > 1
        lens += 1
    assert ax.axon_check_error(err) == (0, 0) and differ == 18


def test_paged_sequences_draw_tokens(ax):
    import synth_inputs as si
    from paper_2608_19889_gb300 import paged
    shape = dict(L=2, D=256, H=8, G=2, d=64, F=512, V=1000, tie=True, bias=False, theta=1e4, eps=1e-5)
    cfg = ax.make_config(shape, 4, 256, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=64, max_prefill_tokens=128)
    m = ax.axon_model_create(cfg, si.make_weights(shape, device=DEV))
    try:
        a = paged.PagedSeqs(m, cfg, 4)
        ids = torch.from_numpy(si.make_ids(1, 40, 1000)).cuda().view(-1)
        greedy, tok = ints(*[0] * 4), ints(*[0] * 4)
        a.extend(ids, [10, 10, 10, 10], next_tokens=greedy)
        temp, top_k, top_p = torch.tensor([0.0, 0.8, 1.2, 1.0], device=DEV), ints(20, 20, 20, 20), torch.full((4,), 0.9, device=DEV)
        r = np.random.default_rng(1)
        tok.copy_(greedy)
        for _ in range(20):
            u = torch.from_numpy(r.random(4, dtype=np.float32)).to(DEV)
            a.sample(tok, u, tok, temperature=temp, top_k=top_k, top_p=top_p)
            assert torch.equal(a.unused[0], tok[0])  # the step's own greedy token
            for i in range(4):
                want = drawn(a.logits[i], float(temp[i]), 20, 0.9, float(u[i]))
                assert want is None or tok[i].item() == want
        a.sample(tok[:2].clone(), u[:2], tok[:2], temperature=temp[:2])  # the first rows alone
        a.check()
        assert a.lengths() == [31, 31, 30, 30]
    finally:
        ax.axon_free(m)


def test_samples_example(ax):
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import samples
    out, prob = samples.generate(steps=40, say=lambda *_: None)
    again, _ = samples.generate(steps=40, say=lambda *_: None)
    other, _ = samples.generate(steps=40, seed=1, say=lambda *_: None)
    assert torch.equal(out, again)  # the same random numbers, the same tokens
    assert torch.equal(out[:, 0], other[:, 0]) and not torch.equal(out[:, 1:], other[:, 1:])
    assert ((prob > 0) & (prob <= 1)).all() and (prob[:, 0] == 1).all()
    with pytest.raises(ValueError):
        samples.generate(steps=samples.CONTEXT)


@pytest.mark.parametrize("H,G,d,B,common,dtype", [(32, 8, 128, 24, 1024, torch.bfloat16), (14, 2, 64, 9, 2000, torch.float16)])
def test_every_step_reads_its_own_tokens(ax, monkeypatch, H, G, d, B, common, dtype):
    """New queries, keys and values each step, launched one after the other and then as a captured step: the attention over shared
    prefixes, whose kernels start before the ones in front have ended, sees them all. Against axon_attn_decode on the same
    cache: both are within 5e-4 max |v| and half a unit of the exact result (values up to 6)."""
    monkeypatch.setenv("AXON_SHARED_MIN_BYTES", "0")
    torch.manual_seed(B)
    steps, whole = 300, common // 16
    per = (common + 2 * steps) // 16 + 2
    k = torch.randn(1, whole + B * (per - whole), G, 16, d, device=DEV).to(dtype)
    cache = ax.make_kv_cache(k, v := torch.randn(k.shape, device=DEV).to(dtype))
    table = torch.empty(B, per, dtype=torch.int32, device=DEV)
    table[:, :whole] = torch.arange(whole, device=DEV)
    table[:, whole:] = whole + torch.arange(B * (per - whole), device=DEV).view(B, -1)
    ctx, rope = ints(*[common] * B), ax.axon_rope_table(per * 16, d, 1e4)
    work, plain = ax.make_shared_workspace(cache, B, H), ax.make_attn_workspace(cache, B, H)
    q, new_k, new_v = (torch.empty(B, n, d, device=DEV, dtype=dtype) for n in (H, G, G))
    a, b, off = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((), device=DEV)
    offsets, prefix = ints(0, B), ints(common)

    def step():
        for t in (q, new_k, new_v):
            t.normal_()
        ax.axon_kv_append(cache, 0, new_k, new_v, ctx, block_table=table, rope=rope, q=q, q_out=q)
        ax.axon_attn_shared(cache, 0, q, ctx, offsets, prefix, a, work, table)
        ax.axon_attn_decode(cache, 0, q, ctx, b, plain, block_table=table)
        torch.maximum(off, ((a.float() - b.float()).abs() - torch.finfo(dtype).eps * b.float().abs()).max(), out=off)
        ctx.add_(1)

    for _ in range(steps):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps):
        graph.replay()
    torch.cuda.synchronize()
    assert v.shape == k.shape and int(ctx[0]) == common + 2 * steps
    assert float(off) <= 6e-3
