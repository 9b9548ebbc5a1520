"""Several continuations of one long prompt: sparse prefill, then decoding from a paged cache.

A prompt goes through `select` and `sparse_attn` layer by layer, its keys and values into the cache;
the cache's slot is forked to one slot per sample, which share the prompt's pages; every step
appends a token per sample and attends with `decode_attn`, which reads the prompt once for all
samples.  The step is captured into a HIP graph and replayed.  Half of the samples then end, the
cache is compacted, and the others go on.

There is no model here: queries, keys and values are random, and stand for what the projections of
a layer would give.  The last step is checked against plain attention over the same tokens.

    python examples/decode_samples.py --tokens 32768 --samples 16 --steps 32
"""
import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

import paper_2502_20766_amd as fpx


def plain_attention(q, k, v):
    """float32 attention of one token: q [Hq, d], k and v [n, Hkv, d]."""
    hq, d = q.shape
    q = q.float().view(k.shape[1], -1, d)
    s = torch.stack([q[h] @ k[:, h].float().T for h in range(k.shape[1])]) / math.sqrt(d)
    p = torch.softmax(s, -1)
    return torch.stack([p[h] @ v[:, h].float() for h in range(k.shape[1])]).view(hq, d)


def run(tokens=8192, samples=8, steps=16, layers=2, heads=32, kv_heads=8, head_dim=128, page=64,
        seed=0, say=print):
    """Runs the example; returns the largest error of the last step."""
    dev, gen = torch.device("cuda"), torch.Generator("cuda").manual_seed(seed)

    def projected(n):
        """Queries, keys and values of n tokens, as one fused projection leaves them."""
        return torch.randn(n, heads + 2 * kv_heads, head_dim, generator=gen, device=dev).bfloat16()

    def split(x):
        return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]

    longest = tokens + 2 * steps
    cache = fpx.Cache(layers, num_pages=-(-longest // page) + samples * (2 * steps // page + 2),
                      num_kv_heads=kv_heads, head_dim=head_dim, num_slots=samples,
                      max_pages=-(-longest // page), page=page)

    # ---- the prompt: sparse prefill, keys and values into slot 0
    fpx.cache_reserve(cache, [0], tokens)
    history = []                                     # for the check at the end
    for layer in range(layers):
        q, k, v = (x.contiguous() for x in split(projected(tokens)))
        lists = fpx.select(q, k, [0, tokens], gamma=0.95, tau=0.1)
        fpx.sparse_attn(q, k, v, lists)              # what the layer goes on with
        fpx.cache_write(cache, layer, k, v, [0], [0, tokens])
        history.append([[k], [v]])

    # ---- one slot per sample; they share the prompt's pages until they write
    if samples > 1:
        fpx.cache_fork(cache, [0] * (samples - 1), np.arange(1, samples, dtype=np.int32))

    def decoder(alive):
        """A graph of one step of the samples in slots `alive`, its input and its outputs."""
        n = len(alive)
        batch = fpx.DecodeBatch(alive, heads, group_start=[0, n], prefix_lens=[tokens])
        rows = np.arange(n + 1, dtype=np.int32)
        x = [projected(n) for _ in range(layers)]
        out = [torch.empty(n, heads, head_dim, dtype=torch.bfloat16, device=dev) for _ in x]
        ws = torch.empty(fpx.cache_workspace_size(cache), dtype=torch.uint8, device=dev)
        attn_ws = torch.empty(fpx.decode_workspace_size(cache, batch), dtype=torch.uint8,
                              device=dev)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fpx.cache_reserve(cache, alive, 1, workspace=ws)
            for layer in range(layers):
                q, k, v = split(x[layer])
                fpx.cache_write(cache, layer, k, v, alive, rows)
                fpx.decode_attn(q, cache, layer, batch, out=out[layer], workspace=attn_ws)
        return graph, x, out

    def decode(alive, keep):
        graph, x, out = decoder(alive)
        begin = time.perf_counter()
        for _ in range(steps):
            for layer in range(layers):
                x[layer].copy_(projected(len(alive)))
                _, k, v = split(x[layer])            # the kept sample's tokens, for the check
                history[layer][0].append(k[keep:keep + 1].clone())
                history[layer][1].append(v[keep:keep + 1].clone())
            graph.replay()
        cache.check()                                # waits; raises if pages had run out
        return x, out, (time.perf_counter() - begin) / steps

    everyone = np.arange(samples, dtype=np.int32)
    x, out, seconds = decode(everyone, samples - 1)
    say(f"{samples} samples of a {tokens}-token prompt, {layers} layers: {seconds * 1e6:.0f} us a "
        f"step, {int(cache.state[0])} pages in use")

    # ---- the first half ends; what they held is given back, the rest moves together
    ended, alive = everyone[:samples // 2], everyone[samples // 2:]
    if len(ended):                                   # of one sample none does
        fpx.cache_free(cache, ended)
    fpx.cache_compact(cache)
    say(f"{len(ended)} samples ended: {int(cache.state[0])} pages in use")
    x, out, seconds = decode(alive, len(alive) - 1)
    say(f"{len(alive)} samples: {seconds * 1e6:.0f} us a step")

    worst = 0.0
    for layer in range(layers):
        k, v = (torch.cat(t) for t in history[layer])
        want = plain_attention(x[layer][-1, :heads], k, v)
        worst = max(worst, float((out[layer][-1].float() - want).abs().max()))
    say(f"last step against plain attention: largest error {worst:.1e}")
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tokens", 32768), ("samples", 16), ("steps", 32), ("layers", 2),
                        ("page", 64), ("seed", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    run(**vars(ap.parse_args()))
