"""Serves a few requests with a small quantized decoder of random weights: prompts of different lengths in one step, then greedy tokens one
step at a time with their log probabilities, a request that ends and one that takes its place, and the score of a given text.

    python examples/serve_decoder.py [--steps 16]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2402_05628_b200 import binding as B  # noqa: E402
from paper_2402_05628_b200.serving import CachedBlock, Decoder, PagedCache, score  # noqa: E402
from workloads import make_block_inputs  # noqa: E402


def build(layers=2, vocab=1000, bits=8, dim=256, heads=4, positions=256, device="cuda:0", seed=0):
    """A decoder in the LLaMA block form, W8A8 (or `bits`), 8-bit cache."""
    sizes = dict(L=positions, D=dim, H=heads, MLP=2 * dim, bits_a=bits, bits_w=bits, bits_p=8, massive=0, outlier_frac=0.0)
    blocks = [CachedBlock(make_block_inputs("c4_llama7b_arch", batch=1, seed=seed + 1 + i, **sizes), device=device) for i in range(layers)]
    rng = np.random.default_rng(seed)
    embedding = torch.from_numpy(rng.standard_normal((vocab, dim)).astype(np.float32)).to(device).to(blocks[0].act_dtype)
    bound = np.full(dim, 4.5, dtype=np.float32)            # a normalised channel stays within some four standard deviations
    return Decoder(blocks, embedding, np.ones(dim, dtype=np.float32), np.zeros(dim, dtype=np.float32), -bound, bound,
                   (0.2 * rng.standard_normal((vocab, dim))).astype(np.float32))


def serve(model, prompts, steps, block_size=16, say=print):
    """Greedy tokens for every prompt: [(tokens, log probabilities)] per request."""
    c, dev = model.blocks[0].cfg, model.embedding.device
    n, longest = len(prompts), max(len(p) for p in prompts) + steps
    cache = PagedCache(len(model.blocks), n * (-(-longest // block_size)), c["H"], block_size, c["D"] // c["H"], n, longest, dev)
    step = cache.plan([len(p) for p in prompts])
    logits = model.forward(torch.tensor([t for p in prompts for t in p], device=dev), step, cache, step.last_rows)
    tokens, logprobs = [], []
    for i in range(steps):
        s = score(logits, top=5)
        tokens.append(s.top_ids[:, 0].clone())
        logprobs.append(s.top_logprobs[:, 0].clone())
        if i + 1 < steps:
            step = cache.plan([1] * n)
            logits = model.forward(tokens[-1], step, cache, step.last_rows)
    t, l = torch.stack(tokens, 1).cpu().tolist(), torch.stack(logprobs, 1).cpu().tolist()
    for r in range(n):
        cache.release(r)
    say("%d requests, %d blocks free again" % (n, cache.free_blocks))
    return list(zip(t, l))


def text_logprobs(model, text, chunk=None, block_size=16):
    """Log probability of every token of a text given those before it (the first has none), the text read in chunks."""
    c, dev = model.blocks[0].cfg, model.embedding.device
    cache = PagedCache(len(model.blocks), -(-len(text) // block_size), c["H"], block_size, c["D"] // c["H"], 1, len(text), dev)
    out = []
    for at in range(0, len(text), chunk or len(text)):
        part = text[at:at + (chunk or len(text))]
        follows = text[at + 1:at + 1 + len(part)]
        follows = follows + [-1] * (len(part) - len(follows))          # (the last token is followed by nothing: padding)
        logits = model.forward(torch.tensor(part, device=dev), cache.plan([len(part)]), cache)
        out.append(score(logits, torch.tensor(follows, dtype=torch.int32, device=dev)).logprob)
    return torch.cat(out)[:len(text) - 1]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=16)
    a = ap.parse_args()
    model = build()
    rng = np.random.default_rng(3)
    prompts = [rng.integers(0, model.vocab, n).tolist() for n in (37, 5, 90, 1)]
    answers = serve(model, prompts, a.steps)
    for p, (t, l) in zip(prompts, answers):
        print("prompt of %2d tokens -> %s   mean log probability %.3f" % (len(p), t[:8], float(np.mean(l))))
    text = prompts[2] + answers[2][0]
    lp = text_logprobs(model, text)
    print("text of %d tokens: perplexity %.1f; of the answer alone %.2f" % (len(text), float(torch.exp(-lp.mean())), float(torch.exp(-lp[len(prompts[2]) - 1:].mean()))))
    assert B.repq_device_status() == 0


if __name__ == "__main__":
    main()
