"""Several samples of one prompt: read once, forked, drawn token by token.

A small random-init decoder reads one prompt; the samples fork from it (they share the prompt's whole blocks) and each draws
its tokens by temperature, top-k and top-p from random numbers of its own. A temperature of 0 gives the greedy
continuation. Run on a GB300:

    python examples/samples.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

SHAPE = dict(L=2, D=256, H=8, G=2, d=64, F=512, V=2000, tie=True, bias=False, theta=1e4, eps=1e-5)
SAMPLES, PROMPT, CONTEXT = 5, 75, 512
TEMPERATURE = [0.0, 0.7, 0.7, 1.0, 1.3]  # of each sample: the first one is greedy


def generate(steps=60, seed=0, say=print):
    """The tokens of every step [steps, SAMPLES] and their probabilities among those that they were drawn from."""
    import torch

    import paper_2608_19889_gb300 as ax
    import synth_inputs as si
    from paper_2608_19889_gb300 import paged

    if not 1 <= steps <= CONTEXT - PROMPT:
        raise ValueError(f"1 .. {CONTEXT - PROMPT} steps are wanted: a sequence ends at {CONTEXT} positions")
    torch.cuda.set_device(0)
    cfg = ax.make_config(SHAPE, SAMPLES, CONTEXT, kv_layout=ax.AXON_KV_PAGED, kv_num_blocks=SAMPLES * CONTEXT // 16,
                         max_prefill_tokens=PROMPT + SAMPLES)
    model = ax.axon_model_create(cfg, si.make_weights(SHAPE, device="cuda"))
    try:
        seqs = paged.PagedSeqs(model, cfg, SAMPLES)
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        prompt = torch.from_numpy(si.make_ids(1, PROMPT, SHAPE["V"])).cuda().view(-1)
        # the prompt but its last token goes to row 0; the other rows get a token each, which the fork replaces
        seqs.extend(torch.cat([prompt[:-1], ints(*range(1, SAMPLES))]), [PROMPT - 1] + [1] * (SAMPLES - 1))
        seqs.fork(ints(*[0] * (SAMPLES - 1)), ints(*range(1, SAMPLES)))
        u = torch.rand(steps, SAMPLES, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
        temperature = torch.tensor(TEMPERATURE, device="cuda")
        top_k, top_p = ints(*[50] * SAMPLES), torch.full((SAMPLES,), 0.95, device="cuda")
        token, prob = prompt[-1:].repeat(SAMPLES), torch.empty(steps, SAMPLES, device="cuda")
        out = torch.empty(steps, SAMPLES, dtype=torch.int32, device="cuda")
        for i in range(steps):
            seqs.sample(token, u[i], out[i], temperature=temperature, top_k=top_k, top_p=top_p, prob=prob[i])
            token = out[i]
        seqs.check()
        for b in range(SAMPLES):
            say(f"temperature {TEMPERATURE[b]}: {out[:12, b].tolist()} ..., mean log-probability {prob[:, b].log().mean():.2f}")
        say(f"lengths {seqs.lengths()}, {seqs.blocks_in_use()} blocks in use")
        return out, prob
    finally:
        ax.axon_free(model)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    generate(ap.parse_args().steps)
