"""Long generation in bounded memory: a sliding window with sinks over a paged cache.

A small random-init decoder reads one prompt, four samples fork from it (they share the prompt's whole blocks), every
sample decodes far past the window while the blocks that slid out go back to the pool, one sample ends, another forks
into its place, and the pool is compacted on the way. Positions are absolute, so a sequence ends at the CONTEXT positions
that the model was made for, however little memory it holds. Run on a GB300:

    python examples/streaming.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

SHAPE = dict(L=2, D=256, H=8, G=2, d=64, F=512, V=2000, tie=True, bias=False, theta=1e4, eps=1e-5, window=96, sinks=4)
SAMPLES, PROMPT, CONTEXT = 4, 75, 4096
POOL = 48  # blocks: 768 tokens for four samples of up to 4096


def generate(steps=300, say=print):
    """The greedy tokens of every step [steps + 1, SAMPLES] and the most blocks that were in use."""
    import torch

    import paper_2608_19889_gb300 as ax
    import synth_inputs as si
    from paper_2608_19889_gb300 import paged

    if PROMPT + steps > CONTEXT:
        raise ValueError(f"at most {CONTEXT - PROMPT} steps: a sequence ends at {CONTEXT} positions")
    torch.cuda.set_device(0)
    cfg = ax.make_config(SHAPE, SAMPLES, CONTEXT, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=POOL,
                         max_prefill_tokens=PROMPT + SAMPLES)
    model = ax.axon_model_create(cfg, si.make_weights(SHAPE, device="cuda"))
    try:
        seqs = paged.PagedSeqs(model, cfg, SAMPLES)
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        prompt = torch.from_numpy(si.make_ids(1, PROMPT, SHAPE["V"])).cuda().view(-1)
        # the prompt goes to row 0; the other rows get a token each, which the fork replaces
        ids = torch.cat([prompt, ints(*range(1, SAMPLES))])
        token = torch.empty(SAMPLES, dtype=torch.int32, device="cuda")
        seqs.extend(ids, [PROMPT] + [1] * (SAMPLES - 1), next_tokens=token)
        seqs.fork(ints(*[0] * (SAMPLES - 1)), ints(*range(1, SAMPLES)))
        seqs.check()
        say(f"prompt of {PROMPT} tokens shared by {SAMPLES} samples: {seqs.blocks_in_use()} blocks")
        token = token[:1].repeat(SAMPLES) + torch.arange(SAMPLES, dtype=torch.int32, device="cuda")  # samples differ
        out, most = [token.clone()], 0
        for i in range(steps):
            if i == steps // 2:  # the last sample ends and the first one forks into its place
                seqs.release(ints(SAMPLES - 1))
                seqs.fork(ints(0), ints(SAMPLES - 1))
                token = torch.cat([token[:-1], token[:1]])
            if i % 64 == 63:
                seqs.compact()
                most = max(most, seqs.blocks_in_use())
                say(f"step {i + 1}: lengths {seqs.lengths()}, {seqs.blocks_in_use()} of {POOL} blocks in use")
            seqs.step(token, next_tokens=token)
            out.append(token.clone())
        seqs.check()
        return torch.stack(out), max(most, seqs.blocks_in_use())
    finally:
        ax.axon_free(model)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=300)
    generate(ap.parse_args().steps)
