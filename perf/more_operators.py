"""The calls between a layer's fused projection and its attention, and the attention of chunks of
new tokens: what a serving loop that takes prompts in chunks runs in every layer.

A case is one pass through one of them.  `op` says which:
  "rotate"  rotate: the heads of queries and keys of `tokens` packed tokens, normed where `norm`
            is true, rotated by their positions.  `seqs` sequences; with `far` 0 their positions
            start at 0 (prompts), else every token has one of its own below `far` (a step);
  "append"  cache_append: the same for the new tokens of a batch, whose keys and values go into a
            paged cache, positions from the lengths that lie there.  `batch` sequences of `old_lo` to
            `old_hi` tokens have got `new_lo` to `new_hi` more;
  "attend"  chunk_attn: the new tokens of every sequence attend to the whole sequence, causally.
            Of the `batch` sequences `singles` have one new token, `idle` hold nothing.

`rotary` elements at the start of a head are rotated, in pairs that `layout` names: "half" (i,
i + rotary / 2) or "interleaved" (2 i, 2 i + 1).  `scaling` names how the frequencies base^(-2 i /
rotary) are stretched by `factor`: "none", "linear" (all of them), "base" (a larger base) or "parts"
(those with less than `high` turns in the original context, and those below `low` wholly).

Keys lie in pages as [layer][page][kv head][token][d], values transposed in steps of 16 tokens,
[layer][page][kv head][token / 16][d][token % 16].
"""
import math
import random

import numpy as np
import torch

own = False

# (query heads, KV heads, head dim), the layers that the other calls are measured on
GEOMETRIES = {
    "llama": (32, 8, 128),     # Llama-3-8B-shaped
    "glm": (32, 2, 128),       # GLM-4-9B-shaped: 16 query heads per KV head
    "qwen": (28, 4, 128),      # Qwen2-7B-shaped: 7 query heads per KV head
    "d64": (64, 16, 64),       # head dim 64, 4 query heads per KV head
    "small": (8, 2, 128),      # one of four tensor-parallel ranks of llama
    "two": (2, 2, 64),         # two heads, no grouping
}

BASE = 500000.0
ORIGINAL = 8192                # tokens of the context that "parts" stretches
LOW, HIGH = 1.0, 32.0
FACTOR = 8.0
EPS = 1e-6


def _rotation(layout, rotary, scaling, norm):
    return {"layout": layout, "rotary": rotary, "scaling": scaling, "norm": norm}


def _rotate(geometry, tokens, seqs, far, layout="half", rotary=128, scaling="none", norm=False):
    return {"op": "rotate", "geometry": geometry, "tokens": tokens, "seqs": seqs, "far": far,
            **_rotation(layout, rotary, scaling, norm)}


def _append(geometry, batch, old_lo, old_hi, new_lo, new_hi, page=64, layout="half", rotary=128,
            scaling="none", norm=False):
    return {"op": "append", "geometry": geometry, "batch": batch, "old_lo": old_lo,
            "old_hi": old_hi, "new_lo": new_lo, "new_hi": new_hi, "page": page,
            **_rotation(layout, rotary, scaling, norm)}


def _attend(geometry, batch, old_lo, old_hi, new_lo, new_hi, singles=0, idle=0, page=64):
    return {"op": "attend", "geometry": geometry, "batch": batch, "old_lo": old_lo,
            "old_hi": old_hi, "new_lo": new_lo, "new_hi": new_hi, "singles": singles,
            "idle": idle, "page": page}


def listed():
    return [
        # the next token of one chat on one of four tensor-parallel ranks: launch and latency
        {"name": "rotate-1", **_rotate("small", 1, 1, 9000, scaling="parts")},
        # a prompt of odd length, half of each head rotated in interleaved pairs
        {"name": "rotate-9001-part", **_rotate("glm", 9001, 1, 0, "interleaved", 64)},
        # the longest packed prompts, with norms of queries and keys
        {"name": "rotate-131072-norm", **_rotate("llama", 131072, 3, 0, scaling="base",
                                                 norm=True)},
        # one decoding step of four short chats
        {"name": "append-4-step", **_append("small", 4, 1, 300, 1, 1, page=16)},
        # one decoding step of 64 sequences with norms, long contexts stretched
        {"name": "append-64-step-norm", **_append("llama", 64, 1, 60000, 1, 1, page=16,
                                                  scaling="parts", norm=True)},
        # chunks of four long prompts, ragged ends
        {"name": "append-4-prompts", **_append("llama", 4, 0, 9000, 7001, 33333)},
        # three short chunks on a small rank: two launches and latency
        {"name": "attend-3-short", **_attend("small", 3, 0, 300, 5, 40, page=16)},
        # a serving batch: most sequences decode, five bring a chunk of their prompt
        {"name": "attend-48-mixed", **_attend("llama", 48, 200, 20000, 200, 1200, singles=43,
                                              idle=1, page=16)},
        # a short question about a very long document
        {"name": "attend-200-of-120k", **_attend("glm", 1, 120000, 120000, 200, 200)},
        # the next chunk of a long prompt, 7 query heads per KV head
        {"name": "attend-2048-of-30k", **_attend("qwen", 1, 30001, 30001, 2048, 2048)},
        # whole prompts of odd lengths from an empty cache, head dim 64
        {"name": "attend-4-prompts-d64", **_attend("d64", 4, 0, 0, 1001, 9001, page=128)},
        # a large chunk at the end of the longest prompt: the products are what costs
        {"name": "attend-4096-of-128k", **_attend("llama", 1, 126976, 126976, 4096, 4096)},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotate", "append", "append", "attend", "attend", "attend"])
    geometry = rng.choice(list(GEOMETRIES))
    hq, hkv, d = GEOMETRIES[geometry]
    page = rng.choice([16, 32, 64, 64, 128, 256])
    turn = _rotation(rng.choice(["half", "half", "interleaved"]),
                     rng.choice([d, d, d // 2, d // 4]),
                     rng.choice(["none", "linear", "base", "parts"]), rng.random() < 0.5)
    if op == "rotate":
        if rng.random() < 0.4:
            return _rotate(geometry, log(1, 256), 1, log(100, 1000000), **turn)
        tokens = log(2, 131072 * 40 * 128 // ((hq + hkv) * d * 2))
        return _rotate(geometry, tokens, min(tokens, rng.randint(1, 8)), 0, **turn)
    if op == "append":
        if rng.random() < 0.4:
            return _append(geometry, log(1, 128), 0, log(2, 16000), 1, log(1, 6), page=page,
                           **turn)
        batch = log(1, 16)
        most = log(30, 90000 // batch)
        return _append(geometry, batch, 0, log(2, 9000), max(1, most // 4), most, page=page,
                       **turn)
    batch = log(1, 64)
    new = log(1, 16384 // batch)
    old = log(2, min(100000, max(50, int(6e12 / (8.0 * hq * d * batch * new))),
                     800000 // batch, int(2e9 / (4 * hkv * d * batch))))
    return _attend(geometry, batch, rng.choice([0, old // 3, old]), old, max(1, new // 3), new,
                   singles=rng.choice([0, 0, batch // 2, batch - 1]), idle=rng.randint(0, batch // 8),
                   page=page)


# ---------------------------------------------------------------- sizes of a case

def _spread(n, lo, hi, salt):
    """n lengths from lo to hi, spread evenly over their logarithm; the case's alone."""
    rng = random.Random(7919 * n + 31 * lo + hi + salt)
    return [min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 1)),
                                                           math.log(hi + 1)))) - (lo == 0))))
            for _ in range(n)]


def _sizes(case):
    """Tokens that each sequence had, and its new ones (an idle one has new rows but no tokens)."""
    old = _spread(case["batch"], case["old_lo"], case["old_hi"], 2)
    new = _spread(case["batch"], case["new_lo"], case["new_hi"], 3)
    if case["op"] == "attend":
        order = list(range(case["batch"]))
        random.Random(case["batch"] * 101 + case["singles"]).shuffle(order)
        for i in order[:case["singles"]]:
            new[i] = 1
    return old, new


def _idle(case):
    return {(i * 13 + 5) % case["batch"] for i in range(case.get("idle", 0))}


def _pages(tokens, page):
    return -(-tokens // page)


# ---------------------------------------------------------------- inputs

def _normal(shape, gen, scale=1.0):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    return x.normal_(0.0, scale, generator=gen)


def _frequencies(case):
    """Radians per position of every pair, in 64 bits on the GPU."""
    r = case["rotary"]
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    base = BASE * FACTOR ** (r / (r - 2)) if case["scaling"] == "base" else BASE
    f = torch.exp(-2 * i / r * math.log(base))
    if case["scaling"] == "linear":
        f = f / FACTOR
    if case["scaling"] == "parts":
        turns = ORIGINAL * f / (2 * math.pi)
        keep = ((turns - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f / FACTOR * (1 - keep) + f * keep
    return f


def _amplitude(case):
    return 0.1 * math.log(FACTOR) + 1 if case["scaling"] == "parts" else 1.0


def _rotation_state(case, gen, rng):
    """Frequencies, norm weights, and the handles that the framework's calls take."""
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    st = {"case": case, "freq": _frequencies(case), "amplitude": _amplitude(case), "wq": None,
          "wk": None}
    if case["norm"]:
        st["wq"], st["wk"] = _normal((2, d), gen, 0.2) + 1
    if own:
        import paper_2502_20766_amd as fpx
        scaled = {} if case["scaling"] == "none" else {
            "scaling": case["scaling"], "factor": FACTOR, "original_len": ORIGINAL,
            "low_turns": LOW, "high_turns": HIGH}
        st["rope"] = fpx.Rope(case["rotary"], base=BASE, layout=case["layout"],
                              amplitude=st["amplitude"], **scaled)
        st["norm"] = fpx.HeadNorm(st["wq"], st["wk"], eps=EPS) if case["norm"] else None
    return st


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    return {"rotate": _prepare_rotate, "append": _prepare_append,
            "attend": _prepare_attend}[case["op"]](case, gen, rng)


def _prepare_rotate(case, gen, rng):
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    T, st = case["tokens"], _rotation_state(case, gen, rng)
    # queries and keys as a fused projection leaves them: one row per token, values behind
    qkv = _normal((T, hq + 2 * hkv, d), gen, 1.5)
    st["q"], st["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]
    if case["far"]:
        pos = rng.integers(0, case["far"], T)
    else:
        cuts = np.sort(rng.permutation(T - 1)[:case["seqs"] - 1] + 1)
        lens = np.diff(np.concatenate([[0], cuts, [T]]))
        pos = np.concatenate([np.arange(n) for n in lens])
    st["pos"] = torch.from_numpy(pos.astype(np.int32)).cuda()
    st["q_out"] = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
    st["k_out"] = torch.empty(T, hkv, d, dtype=torch.bfloat16, device="cuda")
    return st


def _cache_state(st, case, old, new, gen, rng, idle=()):
    """A cache that holds old + new tokens of every sequence on pages in any order."""
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    page, batch = case["page"], case["batch"]
    lens = [0 if i in idle else a + b for i, (a, b) in enumerate(zip(old, new))]
    held = [_pages(n, page) for n in lens]
    pages, slots, wide = sum(held) + 5, batch + 3, max(held) + 1
    table = np.full((slots, wide), -1, np.int32)
    length, ref = np.zeros(slots, np.int32), np.zeros(pages, np.int32)
    free = rng.permutation(pages).astype(np.int32)
    order = rng.permutation(slots)[:batch].astype(np.int32)
    at = 0
    for s, n, m in zip(order, lens, held):
        table[s, :m] = free[at:at + m]
        ref[free[at:at + m]] = 1
        length[s] = n
        at += m
    bits = np.zeros(_pages(pages, 64) * 64, np.uint8)
    bits[:pages] = ref
    state = np.zeros(8, np.int32)
    state[0] = at
    meta = np.concatenate([state, np.packbits(bits, bitorder="little").view(np.int32), length,
                           ref, table.ravel()])
    st["meta"] = torch.from_numpy(meta).cuda()
    st["table"] = torch.from_numpy(table[order].astype(np.int64)).cuda()
    st["k_pool"] = _normal((1, pages, hkv, page, d), gen)
    st["v_pool"] = _normal((1, pages, hkv, page // 16, d, 16), gen)
    st["slots"], st["lens"] = order, lens
    st["cu"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    if own:
        import paper_2502_20766_amd as fpx
        st["cache"] = fpx.Cache(1, pages, hkv, d, slots, wide, page, k=st["k_pool"],
                                v=st["v_pool"], meta=st["meta"])


def _prepare_append(case, gen, rng):
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    old, new = _sizes(case)
    st = _rotation_state(case, gen, rng)
    _cache_state(st, case, old, new, gen, rng)
    T = sum(new)
    qkv = _normal((T, hq + 2 * hkv, d), gen, 1.5)
    st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    st["q_out"] = torch.empty(T, hq, d, dtype=torch.bfloat16, device="cuda")
    seq = np.repeat(np.arange(len(new)), new)
    st["seq"] = torch.from_numpy(seq).cuda()
    st["pos"] = torch.from_numpy(np.concatenate([np.arange(a, a + b)
                                                 for a, b in zip(old, new)])).cuda()
    return st


def _prepare_attend(case, gen, rng):
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    old, new = _sizes(case)
    st = {"case": case}
    idle = _idle(case)
    _cache_state(st, case, old, new, gen, rng, idle)
    # queries with the pull of the first token that long prompts show
    sink = torch.randn(hkv, d, generator=gen, device="cuda")
    sink /= sink.norm(dim=1, keepdim=True)
    q = 1.5 * torch.randn(sum(new), hkv, hq // hkv, d, generator=gen, device="cuda")
    st["q"] = (q + 2.0 * sink[:, None]).reshape(-1, hq, d).bfloat16()
    live = [i for i, n in enumerate(st["lens"]) if n]
    if live:
        st["k_pool"][0, st["table"][live, 0], :, 0] = (3.0 * math.sqrt(d) * sink).bfloat16()
    for i in idle:
        st["slots"][i] = -1
    st["o"] = torch.empty_like(st["q"])
    if own:
        import paper_2502_20766_amd as fpx
        st["batch"] = fpx.ChunkBatch(st["slots"], st["cu"], hq)
        st["ws"] = torch.empty(fpx.chunk_workspace_size(st["cache"], st["batch"]),
                               dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _own_rotate(st):
    import paper_2502_20766_amd as fpx
    return fpx.rotate(st["q"], st["k"], st["pos"], st["rope"], norm=st["norm"],
                      q_out=st["q_out"], k_out=st["k_out"])


def _own_append(st):
    import paper_2502_20766_amd as fpx
    q = fpx.cache_append(st["cache"], 0, st["q"], st["k"], st["v"], st["slots"], st["cu"],
                         st["rope"], norm=st["norm"], q_out=st["q_out"])
    return {"q": q, "k": st["k_pool"], "v": st["v_pool"]}


def _own_attend(st):
    import paper_2502_20766_amd as fpx
    return fpx.chunk_attn(st["q"], st["cache"], 0, st["batch"], out=st["o"], workspace=st["ws"])


def _plain_turn(st, x, weight, pos):
    """Norm and rotation of heads x [T, H, d], in 32 bits, the angles in 64."""
    case = st["case"]
    r, half = case["rotary"], case["rotary"] // 2
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(2, keepdim=True) + EPS) * weight.float()
    angle = pos.double()[:, None] * st["freq"]
    cos = (torch.cos(angle) * st["amplitude"]).float()[:, None]
    sin = (torch.sin(angle) * st["amplitude"]).float()[:, None]
    if case["layout"] == "half":
        u, v = y[..., :half], y[..., half:r]
        turned = [u * cos - v * sin, v * cos + u * sin]
    else:
        u, v = y[..., 0:r:2], y[..., 1:r:2]
        turned = [torch.stack([u * cos - v * sin, v * cos + u * sin], 3).flatten(2)]
    return torch.cat(turned + [y[..., r:]], 2).to(x.dtype)


def _plain_rotate(st):
    st["q_out"].copy_(_plain_turn(st, st["q"], st["wq"], st["pos"]))
    st["k_out"].copy_(_plain_turn(st, st["k"], st["wk"], st["pos"]))
    return st["q_out"], st["k_out"]


def _plain_append(st):
    page, pos = st["case"]["page"], st["pos"]
    st["q_out"].copy_(_plain_turn(st, st["q"], st["wq"], pos))
    p, r = st["table"][st["seq"], pos // page], pos % page
    st["k_pool"][0, p, :, r] = _plain_turn(st, st["k"], st["wk"], pos)
    st["v_pool"][0, p, :, r // 16, :, r % 16] = st["v"]
    return {"q": st["q_out"], "k": st["k_pool"], "v": st["v_pool"]}


def _plain_attend(st):
    hq, hkv, d = GEOMETRIES[st["case"]["geometry"]]
    G, cu, page = hq // hkv, st["cu"], st["case"]["page"]
    for i, n in enumerate(st["lens"]):
        lo, hi = int(cu[i]), int(cu[i + 1])
        if n == 0:
            st["o"][lo:hi] = 0
            continue
        pages = st["table"][i, :_pages(n, page)]
        k = st["k_pool"][0][pages].float().permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n]
        v = st["v_pool"][0][pages].float().permute(1, 0, 2, 4, 3).reshape(hkv, -1, d)[:, :n]
        kt, v = k.transpose(1, 2).contiguous(), v.contiguous()
        key = torch.arange(n, device="cuda")
        step = max(1, 2 ** 29 // (hq * n))           # queries at a time: 2 GB of scores
        for a in range(lo, hi, step):
            b = min(hi, a + step)
            q = st["q"][a:b].float().view(b - a, hkv, G, d).transpose(0, 1) / math.sqrt(d)
            s = (q.reshape(hkv, (b - a) * G, d) @ kt).view(hkv, b - a, G, n)
            last = n - (hi - lo) + torch.arange(a - lo, b - lo, device="cuda")
            s.masked_fill_((key > last[:, None])[:, None], -math.inf)
            s = (s - s.amax(3, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
            total = s.sum(3, keepdim=True)
            o = (s.view(hkv, (b - a) * G, n) @ v).view(hkv, b - a, G, d)
            o = torch.where(total > 0, o / total, 0)
            st["o"][a:b] = o.transpose(0, 1).reshape(b - a, hq, d).to(st["o"].dtype)
    return st["o"]


_PLAIN = {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}
_OWN = {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend}


# ---------------------------------------------------------------- what a pass cannot do without

def _seen(n, m):
    """Pairs of a query and a key that it sees: m new tokens at the end of n."""
    return n * m - m * (m - 1) // 2


def work(case):
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    if case["op"] == "rotate":
        elems = case["tokens"] * (hq + hkv) * d
        return {"bytes": 4 * elems + 4 * case["tokens"],
                "flops": (7 if case["norm"] else 3) * elems}
    old, new = _sizes(case)
    if case["op"] == "append":
        T = sum(new)
        return {"bytes": 4 * T * (hq + 2 * hkv) * d + 4 * len(new),
                "flops": (7 if case["norm"] else 3) * T * (hq + hkv) * d}
    idle = _idle(case)
    both = [(a + b, b) for i, (a, b) in enumerate(zip(old, new)) if i not in idle]
    return {"bytes": 4 * hkv * d * sum(n for n, _ in both) + 4 * sum(new) * hq * d
            + 4 * sum(_pages(n, case["page"]) for n, _ in both),
            "flops": 4 * hq * d * sum(_seen(n, m) for n, m in both)}


# ---------------------------------------------------------------- exact results

def _exact_turn(case, x, weight, pos):
    """Every pair as a complex number times the turn by its position, in 64 bits."""
    r = case["rotary"]
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().sum(2, keepdim=True) / y.shape[2] + EPS)
        y = y * weight.double()
    angle = pos.double()[:, None] * _frequencies(case)
    turn = torch.polar(torch.full_like(angle, _amplitude(case)), angle)[:, None]
    out = y.clone()
    first, second = ((slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half"
                     else (slice(0, r, 2), slice(1, r, 2)))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def exact(case, seed):
    """In 64 bits.  Values that an append moves are copies, which have no other value."""
    st = prepare(case, seed)
    if case["op"] == "rotate":
        return (_exact_turn(case, st["q"], st["wq"], st["pos"]),
                _exact_turn(case, st["k"], st["wk"], st["pos"]))
    if case["op"] == "append":
        k = st["k_pool"].double()
        turned = _exact_turn(case, st["k"], st["wk"], st["pos"])
        for h in range(turned.shape[1]):
            k[0, st["table"][st["seq"], st["pos"] // case["page"]], h,
              st["pos"] % case["page"]] = turned[:, h]
        return {"q": _exact_turn(case, st["q"], st["wq"], st["pos"]), "k": k, "v": None}
    if work(case)["flops"] > 2e13:
        return None
    hq, hkv, d = GEOMETRIES[case["geometry"]]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for i, n in enumerate(st["lens"]):
        if not n:
            continue
        t = torch.arange(n, device="cuda")
        p = st["table"][i][t // case["page"]]
        lo, hi = int(st["cu"][i]), int(st["cu"][i + 1])
        first = n - (hi - lo)                        # position of the first new token
        step = max(1, 2 ** 27 // n)
        for h in range(hq):
            g = h // (hq // hkv)
            key = st["k_pool"][0, p, g, t % case["page"]].double()
            value = st["v_pool"][0, p, g, t % case["page"] // 16, :, t % 16].double()
            for a in range(lo, hi, step):
                b = min(hi, a + step)
                s = st["q"][a:b, h].double() @ key.T / math.sqrt(d)
                see = t <= first + torch.arange(a - lo, b - lo, device="cuda")[:, None]
                s = torch.where(see, s, -math.inf)
                out[a:b, h] = torch.softmax(s, 1) @ value
    return out


if __name__ == "__main__":
    for c in listed():
        print(c["name"], work(c))
