"""The target model's side of a speculative iteration, as measurable cases: what runs between two draft steps.

The draft step reads the target's paged KV cache and emits a block of tokens per request.  The target then takes the block (or a prompt's
next piece) as a chunk of new tokens: it rotates their queries and keys and appends keys and values to the cache, lets every row of the
chunk attend to the cache, and, once the chunk's logits are there, decides how many of the drafted tokens stand and which token follows.

  rope     norm, rotary positions on one or several axes, and the cache write of a ragged chunk   (`hspec_op_chunk_rope_write`)
  attn     attention of a ragged chunk of new tokens over the paged cache                         (`hspec_op_chunk_attention`)
  verify   drafted tokens against the target's probabilities, from given uniform numbers          (`hspec_op_verify`)

Requests are ragged: request b owns rows cu_q[b] .. cu_q[b + 1] - 1 of the chunk, and kv_lens[b] counts its cached tokens with the chunk's
own, so that row i of its n rows stands at cache position kv_lens[b] - n + i.

Head counts, widths, vocabularies, page and block lengths are those of the shapes that this repository is configured for.
"""
import math
import random
import zlib

import torch

own = False

HEADS = {"8b": (32, 8, 128), "32b": (64, 8, 128), "tiny": (4, 2, 64), "mha": (16, 16, 64)}     # query heads, KV heads, head dim
KINDS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------ cases

def _rope(name, heads, kind, batch, new, past, axes=1, norm=True, page=16, pad=0, start=0, layout="sections"):
    return dict(name=name, op="rope", heads=heads, kind=kind, source=kind, batch=batch, new_low=new[0], new_high=new[1], past_low=past[0],
                past_high=past[1], axes=axes, norm=norm, page=page, pad=pad, start=start, layout=layout)


def _attn(name, heads, kind, batch, new, past, window=0, page=16, pad=0):
    return dict(name=name, op="attn", heads=heads, kind=kind, batch=batch, new_low=new[0], new_high=new[1], past_low=past[0],
                past_high=past[1], window=window, page=page, pad=pad)


def _verify(name, batch, block, low, vocab, kind, draft, accept, pruned=0, temperature="one"):
    return dict(name=name, op="verify", batch=batch, block=block, drafts_low=low, vocab=vocab, kind=kind, draft=draft, accept=accept,
                pruned=pruned, temperature=temperature)


def listed():
    return [
        # one request's next token: latency is all there is
        _rope("rope_b1_token", "8b", "bf16", 1, (1, 1), (2048, 2048)),
        # the drafted blocks of a serving batch of odd size, far into long contexts, in a batch padded to a captured graph's size
        dict(_rope("rope_b61_blocks", "tiny", "fp16", 61, (1, 17), (3, 2000), page=8, pad=37, start=900000), source="fp32"),
        # a prompt with pictures: three axes, no norm
        _rope("rope_pictures", "32b", "bf16", 2, (3500, 4700), (0, 300), axes=3, norm=False),
        # one token of one request over a short context: latency again
        _attn("attn_b1_token", "8b", "bf16", 1, (1, 1), (2047, 2047)),
        # verification of a serving batch's blocks
        _attn("attn_b32_blocks", "8b", "bf16", 32, (17, 17), (512, 8192)),
        # the same at high concurrency on the larger shape, ragged blocks, long contexts
        _attn("attn_b64_ragged", "32b", "bf16", 64, (1, 17), (1024, 32000)),
        # odd sizes under a window: heads of 64, fp16, pages of 8, a padded batch
        _attn("attn_b13_window", "mha", "fp16", 13, (1, 300), (0, 5000), window=1000, page=8, pad=5),
        # a prompt's first piece, and the last piece of a long one
        _attn("attn_prompt_8k", "8b", "bf16", 1, (8192, 8192), (0, 0)),
        _attn("attn_piece_of_32k", "32b", "bf16", 1, (1024, 1024), (30777, 30777)),
        # one request's block, drafted by arg-max
        _verify("verify_b1", 1, 16, 16, 128256, "fp32", "argmax", 0.8),
        # a full batch at high concurrency, sampled drafts
        _verify("verify_b128", 128, 16, 16, 152064, "fp32", "sampled", 0.75),
        # 16-bit logits, an odd vocabulary, a drafter over a pruned vocabulary, ragged blocks, greedy and sampling requests mixed
        _verify("verify_b37_pruned", 37, 7, 1, 151937, "bf16", "sampled", 0.6, pruned=32000, temperature="mixed"),
    ]


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    """One more case of the listed ranges (never costlier than the largest listed one)."""
    op = rng.choice(["rope", "attn", "attn", "verify"])
    heads = rng.choice(["8b", "8b", "32b", "32b", "tiny", "mha"])
    kind = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([16, 16, 16, 8, 32, 64, 128])
    if op == "rope":
        batch = _log_int(rng, 1, 64)
        most = max(1, 8192 // batch)
        low = _log_int(rng, 1, most)
        past = _log_int(rng, 1, 8192 // max(1, batch // 8))
        case = _rope(None, heads, kind, batch, (low, _log_int(rng, low, most)), (past // 3, past), axes=rng.choice([1, 1, 2, 3]),
                     norm=rng.random() < 0.6, page=page, pad=rng.choice([0, 0, 9, 40]), start=rng.choice([0, 0, 0, 70000, 1000000]),
                     layout=rng.choice(["sections", "turns"]))
        case["source"] = rng.choice([kind, "fp32"])
    elif op == "attn":
        hq = HEADS[heads][0]
        if rng.random() < 0.6:                      # a batch of single tokens or blocks
            batch, new = _log_int(rng, 1, 64), rng.choice([(1, 1), (1, 9), (8, 8), (17, 17), (1, 33)])
            top = min(32000, int(1.5e9 / (batch * hq * new[1])), 2000000 // batch)
        else:                                       # pieces of prompts
            batch = _log_int(rng, 1, 8)
            high = _log_int(rng, 34, 4096 // batch)
            new = (_log_int(rng, 1, high), high)
            top = max(0, min(32000, int(1.5e9 / (batch * hq * high)) - high))
        high = _log_int(rng, 1, max(1, top))
        case = _attn(None, heads, kind, batch, new, (rng.choice([0, high // 8, high]), high), window=rng.choice([0, 0, 0, 2048, 333]),
                     page=page, pad=rng.choice([0, 0, 3, 64]))
    else:
        block = rng.randint(1, 32)
        vocab = rng.choice([32000, 128256, 151936, 152064, rng.randint(1000, 152064)])
        batch = _log_int(rng, 1, min(256, 3 * 10**8 // (block + 1) // vocab))
        draft = rng.choice(["sampled", "sampled", "argmax"])
        case = _verify(None, batch, block, rng.randint(0, block), vocab, rng.choice(["fp32", "fp32", "bf16", "fp16"]), draft,
                       rng.choice([0.3, 0.6, 0.8, 0.95]), pruned=rng.choice([0, 0, vocab // 4]) if draft == "sampled" else 0,
                       temperature=rng.choice(["one", "mixed", "mixed"]))
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + zlib.crc32(what.encode())) % (1 << 62))
    return g


def _randn(seed, what, shape, kind=torch.float32, std=1.0):
    return torch.empty(shape, dtype=kind, device="cuda").normal_(0.0, std, generator=_gen(seed, what))


def _rand(seed, what, shape):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(0.0, 1.0, generator=_gen(seed, what))


def _spread(n, low, high):
    """n whole numbers from low to high: evenly spaced quantiles of a log-uniform distribution, so that every seed has the same set."""
    a, b = math.log(low + 1), math.log(high + 1)
    return [min(high, max(low, int(round(math.exp(a + (b - a) * ((i + 0.5) / n if n > 1 else 1.0)) - 1)))) for i in range(n)]


def _lengths(case):
    """New tokens and earlier tokens of every request, the same for every seed."""
    n = case["batch"]
    new, past = _spread(n, case["new_low"], case["new_high"]), _spread(n, case["past_low"], case["past_high"])
    random.Random(n * 7919 + case["new_high"]).shuffle(new)
    random.Random(n * 104729 + case["past_high"]).shuffle(past)
    return new, past


def _layout(case, seed):
    """The chunk's rows and the cache's pages: a shuffled page table whose unused entries name no page."""
    new, past = _lengths(case)
    kv = [a + b for a, b in zip(new, past)]
    pages = [-(-c // case["page"]) for c in kv]
    perm = torch.randperm(sum(pages) + 2, generator=_gen(seed, "pages"), device="cuda").to(torch.int32).cpu()
    table = torch.full((len(kv), max(pages) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return dict(case=case, table=table.cuda(), cu_q=torch.tensor(starts, dtype=torch.int32, device="cuda"), pages=perm.numel(),
                kv_lens=torch.tensor(kv, dtype=torch.int32, device="cuda"), rows=starts[-1], rows_padded=starts[-1] + case["pad"],
                new_high=max(new), kv_high=max(kv))


def _positions(case, lay, seed):
    """Rotary positions [axes, rows]: text counts up on every axis alike; with several axes the last two thirds of a request's rows are a
    picture, whose rows count along the second and third axis from the position where the text ended."""
    new, past = _lengths(case)
    shift = random.Random(int(seed)).randrange(64)
    every = []
    for n, p in zip(new, past):
        i = torch.arange(n, dtype=torch.int64)
        base = case["start"] + p + shift
        pos = (base + i).repeat(case["axes"], 1)
        if case["axes"] > 1:
            text, wide = n // 3, 1 + int(math.isqrt(n))
            j = torch.clamp(i - text, min=0)
            for axis in range(case["axes"]):
                step = torch.zeros_like(j) if axis == 0 else j // wide if axis == 1 else j % wide
                pos[axis] = torch.where(i < text, base + i, base + text + step)
        every.append(pos)
    pos = torch.cat(every + [torch.zeros((case["axes"], case["pad"]), dtype=torch.int64)], dim=1)
    return pos.to(torch.int32).cuda().contiguous()


def _pair_axes(case):
    """Which axis each of the head's rotated pairs follows: in sections (1/4, 3/8, 3/8 of the pairs for three axes), or by turns."""
    pairs, axes = HEADS[case["heads"]][2] // 2, case["axes"]
    if case["layout"] == "turns":
        return [j % axes for j in range(pairs)]
    if axes == 3:
        return [0] * (pairs // 4) + [1] * (3 * pairs // 8) + [2] * (pairs - pairs // 4 - 3 * pairs // 8)
    return [j * axes // pairs for j in range(pairs)]


def _logits(seed, what, rows, vocab):
    """Logits as a language model has them: a wide bulk, and a few tokens far above it."""
    z = _randn(seed, what, (rows, vocab), std=2.0)
    top = torch.randint(0, vocab, (rows, 6), generator=_gen(seed, what + "top"), device="cuda")
    z.scatter_(1, top, 9.0 + 7.0 * _rand(seed, what + "lead", (rows, 6)))
    return z


def _drafts(case):
    """Drafted tokens that are put to the target, for every request."""
    n = [case["drafts_low"] + (i * (case["block"] - case["drafts_low"]) + case["batch"] // 2) // max(1, case["batch"] - 1) for i in range(case["batch"])]
    return [min(case["block"], x) for x in n]


def _prepare_verify(case, seed):
    B, k, V, Vd = case["batch"], case["block"], case["vocab"], case["pruned"] or case["vocab"]
    n = _drafts(case)
    random.Random(B * 31 + k).shuffle(n)
    starts = [0]
    for x in n:
        starts.append(starts[-1] + x + 1)
    T = starts[-1]
    vocab_map = None
    if case["pruned"]:
        vocab_map = torch.sort(torch.randperm(V, generator=_gen(seed, "map"), device="cuda")[:Vd])[0]
    zd = _logits(seed, "draft", B * k, Vd)
    zt = _logits(seed, "target", T, V)
    # where the drafter is right the target's logits are the drafter's with a little noise; else they are another model's
    row = torch.cat([torch.arange(s, s + x, device="cuda") for s, x in zip(starts, n)]) if sum(n) else torch.empty(0, dtype=torch.int64, device="cuda")
    src = torch.cat([torch.arange(b * k, b * k + x, device="cuda") for b, x in enumerate(n)]) if sum(n) else row
    right = _rand(seed, "right", (row.numel(),)) < case["accept"]
    row, src = row[right], src[right]
    if vocab_map is None:
        zt[row] = zd[src] + 0.1 * zt[row].clamp(-4, 4)
    else:
        zt[row] = zt[row].clamp(-4, 4)
        zt[row.unsqueeze(1), vocab_map] = zd[src] + 0.1 * zt[row.unsqueeze(1), vocab_map]
    kind = KINDS[case["kind"]]
    zd, zt = zd.to(kind), zt.to(kind)
    warm = torch.ones(B, device="cuda")
    if case["temperature"] == "mixed":
        warm = torch.tensor([1.0, 0.0, 0.7, 1.3], device="cuda").repeat(-(-B // 4))[:B].contiguous()
    if case["draft"] == "argmax":
        ids = torch.argmax(zd, dim=1).reshape(B, k)
    else:
        ids = torch.empty((B, k), dtype=torch.int64, device="cuda")
        for b in range(B):
            q = torch.softmax(zd[b * k:(b + 1) * k].float() / max(float(warm[b]), 1e-3), dim=1)
            ids[b] = torch.multinomial(q, 1, generator=_gen(seed, "ids%d" % b)).squeeze(1)
    if vocab_map is not None:
        ids = vocab_map[ids]
    state = dict(case=case, target=zt, draft=None if case["draft"] == "argmax" else zd.reshape(B, k, Vd), ids=ids.to(torch.int32).contiguous(),
                 cu_q=torch.tensor(starts, dtype=torch.int32, device="cuda"), map=None if vocab_map is None else vocab_map.to(torch.int32),
                 temperature=warm, alpha=_rand(seed, "alpha", (B, k)), u=_rand(seed, "u", (B,)),
                 n_accept=torch.empty(B, dtype=torch.int32, device="cuda"), tokens=torch.empty((B, k + 1), dtype=torch.int32, device="cuda"))
    if own:                                                        # the scratch that the caller of this library owns
        import paper_2609_24197_b200 as hs
        state["workspace"] = torch.empty(hs.hspec_verify_workspace_bytes(B, k), dtype=torch.uint8, device="cuda")
    return state


def prepare(case, seed):
    if case["op"] == "verify":
        return _prepare_verify(case, seed)
    hq, hkv, dh = HEADS[case["heads"]]
    kind = KINDS[case["kind"]]
    s = _layout(case, seed)
    pool = (s["pages"], case["page"], hkv, dh)
    s["k_pool"], s["v_pool"] = _randn(seed, "k", pool, kind), _randn(seed, "v", pool, kind)
    if case["op"] == "rope":
        s["qkv"] = _randn(seed, "qkv", (s["rows_padded"], (hq + 2 * hkv) * dh), KINDS[case["source"]])
        s["pos"], s["pair_axis"] = _positions(case, s, seed), bytes(_pair_axes(case))
        s["q_norm"] = 1.0 + _randn(seed, "qn", (dh,), std=0.1) if case["norm"] else None
        s["k_norm"] = 1.0 + _randn(seed, "kn", (dh,), std=0.1) if case["norm"] else None
        s["q"] = torch.zeros((s["rows_padded"], hq, dh), dtype=kind, device="cuda")
        return s
    # queries a little larger than unit length, as after a norm with weights above one: scores then spread over a few units
    s["q"] = _randn(seed, "q", (s["rows_padded"], hq, dh), kind, std=1.5)
    s["o"] = torch.zeros((s["rows_padded"], hq, dh), dtype=kind, device="cuda")
    if own:                                                        # the scratch that the caller of this library owns
        import paper_2609_24197_b200 as hs
        s["workspace"] = torch.empty(hs.hspec_chunk_attention_workspace_bytes(hq, hkv, dh), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass

THETA, EPS = 1.0e6, 1e-6


def _places(s):
    """Request, index within its chunk, cache position and cache slot of every row."""
    rows = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(s["cu_q"].long(), rows, right=True) - 1
    i = rows - s["cu_q"].long()[b]
    at = (s["kv_lens"] - (s["cu_q"][1:] - s["cu_q"][:-1])).long()[b] + i
    page = s["case"]["page"]
    return b, i, at, s["table"].long()[b, at // page] * page + at % page


def _plain_rope(s):
    hq, hkv, dh = HEADS[s["case"]["heads"]]
    n, half = s["rows"], dh // 2
    x = s["qkv"][:n].float().reshape(n, hq + 2 * hkv, dh)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if s["q_norm"] is not None:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * s["q_norm"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * s["k_norm"]
    rate = float(THETA) ** (-2.0 * torch.arange(half, dtype=torch.float64, device="cuda") / dh)
    axis = torch.tensor(list(s["pair_axis"]), device="cuda")
    angle = s["pos"][:, :n].double()[axis].T * rate                # [rows, pairs]: far positions times rates need 64 bits
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)

    def turned(y):
        a, b = y[..., :half], y[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)

    slot = _places(s)[3]
    s["q"][:n] = turned(q).to(s["q"].dtype)
    s["k_pool"].view(-1, hkv, dh)[slot] = turned(k).to(s["q"].dtype)
    s["v_pool"].view(-1, hkv, dh)[slot] = v.to(s["q"].dtype)
    return dict(q=s["q"], k_pool=s["k_pool"], v_pool=s["v_pool"])


def _plain_attn(s):
    hq, hkv, dh = HEADS[s["case"]["heads"]]
    case, rep, n, L = s["case"], hq // hkv, s["new_high"], s["kv_high"]
    key = torch.arange(L, device="cuda")
    slot = s["table"].long().clamp(min=0)[:, key // case["page"]] * case["page"] + key % case["page"]         # [B, L]
    there = key < s["kv_lens"].unsqueeze(1)

    def cached(pool):                                              # [B, kv heads, L, dh]
        return (pool.view(-1, hkv, dh)[slot].float() * there[:, :, None, None]).transpose(1, 2)

    b, i, at, _ = _places(s)
    q = torch.zeros((case["batch"], n, hq, dh), device="cuda")
    q[b, i] = s["q"][:s["rows"]].float()
    q = q.reshape(case["batch"], n, hkv, rep, dh).permute(0, 2, 1, 3, 4).reshape(case["batch"], hkv, n * rep, dh)
    score = torch.matmul(q, cached(s["k_pool"]).transpose(2, 3)).reshape(case["batch"], hkv, n, rep, L)
    place = torch.full((case["batch"], n), -1, dtype=torch.int64, device="cuda")
    place[b, i] = at
    seen = key <= place.unsqueeze(2)
    if case["window"]:
        seen &= key > place.unsqueeze(2) - case["window"]
    score.mul_(dh ** -0.5).masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    score.sub_(score.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = score.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(score.reshape(case["batch"], hkv, n * rep, L), cached(s["v_pool"])).reshape(case["batch"], hkv, n, rep, dh) / total
    o = o.permute(0, 2, 1, 3, 4).reshape(case["batch"], n, hq, dh)
    s["o"][:s["rows"]] = o[b, i].to(s["o"].dtype)
    return s["o"]


def _softmax64(z, temperature):
    """Probabilities in 64 bits (a cumulative sum over the vocabulary, and values next to a uniform number, need them); at temperature 0
    all of it goes to the first of the largest."""
    z = z.double()
    e = torch.exp((z - z.amax(-1, keepdim=True)) / temperature.double().clamp(min=1e-30))
    p = e / e.sum(-1, keepdim=True)
    first = torch.argmax(z, dim=-1, keepdim=True)
    return torch.where(temperature > 0, p, torch.zeros_like(p).scatter_(-1, first, 1.0))


def _plain_verify(s):
    B, k, V = s["case"]["batch"], s["case"]["block"], s["case"]["vocab"]
    cu, ids = s["cu_q"].long(), s["ids"].long()
    drafts = torch.clamp(cu[1:] - cu[:-1] - 1, max=k)
    i = torch.arange(k, device="cuda")
    put = i < drafts.unsqueeze(1)
    of = torch.searchsorted(cu, torch.arange(s["target"].shape[0], device="cuda"), right=True) - 1
    p = _softmax64(s["target"], s["temperature"][of].unsqueeze(1))
    row = torch.where(put, cu[:-1].unsqueeze(1) + i, cu[:-1].unsqueeze(1))
    px = p[row, ids]
    warm = (s["temperature"] > 0).unsqueeze(1)
    if s["draft"] is None:
        q, qx = None, torch.ones_like(px)
    else:
        q = _softmax64(s["draft"], s["temperature"][:, None, None])
        qx = torch.gather(q, 2, (ids if s["map"] is None else torch.searchsorted(s["map"].long(), ids)).unsqueeze(2)).squeeze(2)
        qx = torch.where(warm, qx, torch.ones_like(qx))
    taken = (px > 0) & (torch.clamp(px / qx, max=1.0) >= s["alpha"].double()) & put
    n = torch.cumprod(taken.long(), dim=1).sum(1)
    rest = p[cu[:-1] + n]
    b, at, cut = torch.arange(B, device="cuda"), torch.clamp(n, max=k - 1), ((n < drafts) & warm.squeeze(1)).unsqueeze(1)
    if q is None:
        less = torch.zeros_like(rest).scatter_(1, ids[b, at].unsqueeze(1), float("inf"))
    elif s["map"] is None:
        less = q[b, at]
    else:
        less = torch.zeros_like(rest)
        less[:, s["map"].long()] = q[b, at]
    rest = torch.where(cut, torch.clamp(rest - less, min=0.0), rest)
    upto = torch.cumsum(rest, dim=1)
    new = (upto <= s["u"].double().unsqueeze(1) * upto[:, -1:]).sum(1).clamp(max=V - 1)
    j = torch.arange(k + 1, device="cuda")
    tokens = torch.where(j < n.unsqueeze(1), torch.nn.functional.pad(ids, (0, 1)), torch.where(j == n.unsqueeze(1), new.unsqueeze(1), -1))
    s["n_accept"].copy_(n)
    s["tokens"].copy_(tokens)
    return dict(n_accept=s["n_accept"], tokens=s["tokens"])


def run(s):
    case = s["case"]
    if not own:
        return {"rope": _plain_rope, "attn": _plain_attn, "verify": _plain_verify}[case["op"]](s)
    import paper_2609_24197_b200 as hs
    if case["op"] == "rope":
        hs.hspec_op_chunk_rope_write(s["qkv"], s["pos"], s["pair_axis"], s["cu_q"], s["kv_lens"], s["table"], s["q"], s["k_pool"], s["v_pool"],
                                     THETA, q_norm_w=s["q_norm"], k_norm_w=s["k_norm"], eps=EPS)
        return dict(q=s["q"], k_pool=s["k_pool"], v_pool=s["v_pool"])
    if case["op"] == "attn":
        hs.hspec_op_chunk_attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["cu_q"], s["kv_lens"], s["o"], s["workspace"],
                                    window=case["window"])
        return s["o"]
    hs.hspec_op_verify(s["target"], s["draft"], s["ids"], s["alpha"], s["u"], s["n_accept"], s["tokens"], s["workspace"], cu_q=s["cu_q"],
                       vocab_map=s["map"], temperature=s["temperature"])
    return dict(n_accept=s["n_accept"], tokens=s["tokens"])


# ------------------------------------------------------------------------------------------------ accounting

def _pairs(n, past, window):
    """Visible (row, key) pairs of one request's head, and the keys that any of its rows sees."""
    if not window:
        return n * past + n * (n + 1) // 2, n + past
    return sum(min(past + i + 1, window) for i in range(n)), min(n + past, window + n - 1)


def work(case):
    if case["op"] == "verify":
        # a request's rows up to its first refused draft decide; how many those are on average follows from the share of right drafts
        take = 0.93 * case["accept"]
        n = _drafts(case)
        target = sum(sum(take ** i for i in range(x + 1)) for x in n)
        draft = 0.0 if case["draft"] == "argmax" else sum(sum(take ** i for i in range(x)) for x in n)
        if case["temperature"] == "mixed":
            draft *= 0.75                                          # greedy requests need the target's rows alone
        values = target * case["vocab"] + draft * (case["pruned"] or case["vocab"])
        return {"bytes": values * BYTES[case["kind"]] + 16.0 * case["batch"] * case["block"], "flops": 3.0 * values}
    hq, hkv, dh = HEADS[case["heads"]]
    new, past = _lengths(case)
    rows = float(sum(new))
    if case["op"] == "rope":
        values = rows * (hq + 2 * hkv) * dh
        return {"bytes": values * (BYTES[case["source"]] + 2) + 4.0 * rows * case["axes"], "flops": 3.0 * values}
    seen = [_pairs(n, p, case["window"]) for n, p in zip(new, past)]
    return {"bytes": 4.0 * hkv * dh * sum(k for _, k in seen) + 4.0 * rows * hq * dh, "flops": 4.0 * hq * dh * float(sum(p for p, _ in seen))}


# ------------------------------------------------------------------------------------------------ by the definitions, in 64 bits

def _exact_rope(s):
    case = s["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    n, half = s["rows"], dh // 2
    x = s["qkv"].double().view(-1, hq + 2 * hkv, dh)[:n].clone()
    for first, count, w in ((0, hq, s["q_norm"]), (hq, hkv, s["k_norm"])):
        part = x[:, first:first + count]
        if w is not None:
            part = part / torch.sqrt(torch.mean(part ** 2, dim=2, keepdim=True) + EPS) * w.double()
        turn = torch.empty((n, half), dtype=torch.complex128, device="cuda")
        for j, axis in enumerate(s["pair_axis"]):
            a = s["pos"][axis, :n].double() * math.exp(-2.0 * j / dh * math.log(THETA))
            turn[:, j] = torch.polar(torch.ones_like(a), a)
        z = torch.complex(part[..., :half].contiguous(), part[..., half:].contiguous()) * turn[:, None, :]
        x[:, first:first + count] = torch.cat([z.real, z.imag], dim=2)
    q, kp, vp = s["q"].double(), s["k_pool"].double(), s["v_pool"].double()
    q[:n] = x[:, :hq]
    cu, kv, table = s["cu_q"].tolist(), s["kv_lens"].tolist(), s["table"].cpu()
    for b in range(case["batch"]):
        m = cu[b + 1] - cu[b]
        at = torch.arange(kv[b] - m, kv[b])
        page, off = table[b].long()[at // case["page"]].cuda(), (at % case["page"]).cuda()
        kp[page, off] = x[cu[b]:cu[b + 1], hq:hq + hkv]
        vp[page, off] = x[cu[b]:cu[b + 1], hq + hkv:]
    return dict(q=q, k_pool=kp, v_pool=vp)


def _exact_attn(s):
    case = s["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    out = s["o"].double()
    cu, kv = s["cu_q"].tolist(), s["kv_lens"].tolist()
    for b in range(case["batch"]):
        n, L = cu[b + 1] - cu[b], kv[b]
        pages = s["table"][b, :-(-L // case["page"])].long()
        K, V = (p[pages].reshape(-1, hkv, dh)[:L].double() for p in (s["k_pool"], s["v_pool"]))
        at = torch.arange(L - n, L, device="cuda").unsqueeze(1)
        far = at - torch.arange(L, device="cuda")
        hidden = (far < 0) if not case["window"] else (far < 0) | (far >= case["window"])
        for h in range(hq):
            z = (s["q"][cu[b]:cu[b + 1], h].double() @ K[:, h // (hq // hkv)].T) / math.sqrt(dh)
            out[cu[b]:cu[b + 1], h] = torch.softmax(z.masked_fill(hidden, -math.inf), dim=1) @ V[:, h // (hq // hkv)]
    return out


def _exact_verify(s):
    case = s["case"]
    B, k, V = case["batch"], case["block"], case["vocab"]
    cu, ids, warm = s["cu_q"].tolist(), s["ids"].long().tolist(), s["temperature"].double().tolist()
    counts, tokens = torch.zeros(B, dtype=torch.int32), torch.full((B, k + 1), -1, dtype=torch.int32)

    def share(z, t):
        if t == 0:
            return torch.zeros_like(z).index_fill_(0, torch.argmax(z), 1.0)
        w = z / t
        return torch.exp(w - torch.logsumexp(w, 0))

    for b in range(B):
        n = min(k, cu[b + 1] - cu[b] - 1)
        alpha = s["alpha"][b].double().tolist()
        rest = None
        for i in range(n):
            p = share(s["target"][cu[b] + i].double(), warm[b])
            x = ids[b][i]
            q = torch.zeros_like(p)
            if s["draft"] is None or warm[b] == 0:
                q[x] = 1.0
            elif s["map"] is None:
                q = share(s["draft"][b, i].double(), warm[b])
            else:
                q[s["map"].long()] = share(s["draft"][b, i].double(), warm[b])
            if float(p[x]) > 0 and min(1.0, float(p[x]) / float(q[x])) >= alpha[i]:
                counts[b] += 1
                tokens[b, i] = x
                continue
            rest = p if warm[b] == 0 else torch.relu(p - q)
            break
        if rest is None:
            rest = share(s["target"][cu[b] + n].double(), warm[b])
        upto = torch.cumsum(rest, 0)
        tokens[b, int(counts[b])] = int(torch.searchsorted(upto, s["u"][b].double() * upto[-1], right=True).clamp(max=V - 1))
    return dict(n_accept=counts, tokens=tokens)


def exact(case, seed):
    return {"rope": _exact_rope, "attn": _exact_attn, "verify": _exact_verify}[case["op"]](prepare(case, seed))
