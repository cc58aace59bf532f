"""More of the target model's side of a speculative iteration, as measurable cases: a hybrid target's recurrent layers, and its logits.

A target that mixes Mamba layers with attention carries a state instead of a cache.  Like the attention's cache it is read and advanced by a ragged
chunk of new tokens (a prompt's piece, a drafted block, a single token), and after a verification it stands behind the accepted tokens alone.
Between the target's LM head and the verification stand the rules that a request brings along: penalties for what was said before, biases,
and a grammar's allowed tokens.

  scan     short causal convolution, selective scan and gate of a ragged chunk, with carried states    (`hspec_op_chunk_scan`)
  logits   penalties for repeated tokens, biases and allowed tokens, row by row of a drafted block      (`hspec_op_adjust_logits`)

Requests are ragged: request b owns rows cu_q[b] .. cu_q[b + 1] - 1 of the chunk.

Widths, head counts, vocabularies and block lengths are those of the shapes that this repository is configured for.
"""
import math
import random
import zlib

import torch

own = False

SHAPES = {"8b": (8192, 64, 128, 4), "32b": (10240, 64, 128, 4), "tiny": (512, 64, 16, 1), "odd": (960, 40, 24, 3)}     # Di, head width, state, groups
KINDS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
TAPS = 4                                                           # of the convolution, the token's own among them


# ------------------------------------------------------------------------------------------------ cases

def _scan(name, shape, kind, batch, new, mode="step", fresh="none", out=None, pad=0, dt="columns", tokens=0):
    """mode: "step" keeps the state behind every row, "look" (a verification's pass) keeps none of them, "commit" (what follows it) computes no
    outputs and keeps the accepted rows' state.  `tokens`: requests of a single token next to the others."""
    return dict(name=name, op="scan", shape=shape, kind=kind, out=out or kind, batch=batch, new_low=new[0], new_high=new[1], mode=mode, fresh=fresh,
                pad=pad, dt=dt, tokens=tokens)


def _logits(name, batch, rows, vocab, kind, history, out=None, penalties=True, biases=0, grammar="none", place="apart", pad=0):
    return dict(name=name, op="logits", batch=batch, rows_low=rows[0], rows_high=rows[1], vocab=vocab, kind=kind, out=out or kind,
                history_low=history[0], history_high=history[1], penalties=penalties, biases=biases, grammar=grammar, place=place, pad=pad)


def listed():
    return [
        # one request's next token: latency is all there is
        _scan("scan_b1_token", "8b", "bf16", 1, (1, 1)),
        # a serving batch's next tokens: every state is read and written once
        _scan("scan_b64_tokens", "32b", "bf16", 64, (1, 1)),
        # verification of drafted blocks: outputs, and no state kept; then what the accepted tokens add to the state
        _scan("scan_b32_look", "8b", "bf16", 32, (17, 17), mode="look"),
        _scan("scan_b61_commit", "32b", "fp16", 61, (1, 17), mode="commit", pad=37),
        # a whole prompt, and pieces of prompts of any length next to other requests' tokens
        _scan("scan_prompt_8k", "8b", "bf16", 1, (8192, 8192), fresh="all"),
        _scan("scan_pieces", "32b", "fp16", 5, (150, 2500), fresh="some", pad=3, tokens=12),
        # small states, 32-bit rows, dt from a projection of its own
        _scan("scan_tiny_ragged", "tiny", "fp32", 29, (1, 700), fresh="some", dt="apart", pad=5),
        # one request's next token with penalties: latency again
        _logits("logits_b1", 1, (1, 1), 128256, "fp32", (2048, 2048)),
        # drafted blocks of a serving batch with everything on
        _logits("logits_b32_rules", 32, (17, 17), 128256, "bf16", (512, 8192), out="fp32", biases=40, grammar="some"),
        # high concurrency
        _logits("logits_b128", 128, (17, 17), 152064, "fp32", (1024, 32768)),
        # a grammar alone, in place, over an odd vocabulary
        _logits("logits_grammar", 37, (1, 9), 151937, "fp16", (0, 300), penalties=False, grammar="all", place="same", pad=11),
    ]


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    """One more case of the listed ranges (never costlier than the largest listed one)."""
    if rng.random() < 0.6:
        shape = rng.choice(["8b", "8b", "32b", "32b", "tiny", "odd"])
        kind = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        tokens = 0
        if rng.random() < 0.6:                      # single tokens and blocks
            batch, new = _log_int(rng, 1, 61), rng.choice([(1, 1), (1, 9), (8, 8), (17, 17), (1, 17), (1, 33)])
            mode = rng.choice(["step", "look", "commit"])
        else:                                       # prompts and pieces of them
            batch = _log_int(rng, 1, 8)
            high = _log_int(rng, 34, 8192 // batch)
            new, mode = (_log_int(rng, 1, high), high), "step"
            tokens = rng.choice([0, 0, rng.randint(1, 12)]) if batch * high < 6000 else 0
        case = _scan(None, shape, kind, batch, new, mode=mode, fresh=rng.choice(["none", "some", "all"]), pad=rng.choice([0, 0, 3, 40]),
                     out=rng.choice([kind, kind, "fp32"]), dt=rng.choice(["columns", "columns", "apart"]), tokens=tokens)
    else:
        vocab = rng.choice([32000, 128256, 151936, 152064, rng.randint(1000, 152064)])
        rows = rng.choice([(1, 1), (1, 1), (1, 9), (17, 17), (1, 33)])
        batch = _log_int(rng, 1, max(1, min(200, 3 * 10**8 // rows[1] // vocab)))
        high = _log_int(rng, 1, 32768)
        place = rng.choice(["apart", "apart", "apart", "same"])
        kind = rng.choice(["fp32", "fp32", "bf16", "fp16"])
        case = _logits(None, batch, rows, vocab, kind, (rng.choice([0, high // 8, high]), high), out=rng.choice([kind, kind, "fp32"]) if place == "apart" else kind,
                       penalties=place == "apart" and rng.random() < 0.8, biases=rng.choice([0, 0, 1, 300]) if place == "apart" else 0,
                       grammar="all" if place == "same" else rng.choice(["none", "some", "all"]), place=place, pad=rng.choice([0, 0, 7]))
        if case["biases"] == 0 and case["grammar"] == "none":
            case["penalties"] = True
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + zlib.crc32(what.encode())) % (1 << 62))
    return g


def _randn(seed, what, shape, kind=torch.float32, std=1.0):
    return torch.empty(shape, dtype=kind, device="cuda").normal_(0.0, std, generator=_gen(seed, what))


def _rand(seed, what, shape, low=0.0, high=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").uniform_(low, high, generator=_gen(seed, what))


def _spread(n, low, high):
    """n whole numbers from low to high: evenly spaced quantiles of a log-uniform distribution, so that every seed has the same set."""
    a, b = math.log(low + 1), math.log(high + 1)
    got = [min(high, max(low, int(round(math.exp(a + (b - a) * ((i + 0.5) / n if n > 1 else 1.0)) - 1)))) for i in range(n)]
    random.Random(n * 7919 + high).shuffle(got)
    return got


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _rows_of(case):
    """Rows of every request, the same for every seed."""
    if case["op"] == "logits":
        return _spread(case["batch"], case["rows_low"], case["rows_high"])
    new = _spread(case["batch"], case["new_low"], case["new_high"]) + [1] * case["tokens"]
    random.Random(len(new)).shuffle(new)
    return new


def _fresh_of(case):
    n = case["batch"] + case["tokens"]
    return [1 if case["fresh"] == "all" or (case["fresh"] == "some" and b % 3 == 1) else 0 for b in range(n)]


def _kept_of(case):
    """Rows whose state is kept: all of them, none, or the accepted drafts and the token in front of them."""
    new = _rows_of(case)
    if case["mode"] == "step":
        return new
    return [0] * len(new) if case["mode"] == "look" else [1 + (b * 5 + 3) % n for b, n in enumerate(new)]


def _prepare_scan(case, seed):
    Di, P, N, G = SHAPES[case["shape"]]
    H, xbc, new, kind = Di // P, Di + 2 * G * N, _rows_of(case), KINDS[case["kind"]]
    B, T = len(new), sum(new)
    rows = T + case["pad"]
    wide = Di + xbc + (H if case["dt"] == "columns" else 0)
    x = _randn(seed, "x", (rows, wide), kind)
    s = dict(case=case, new=new, x=x, dt=None if case["dt"] == "columns" else _randn(seed, "dt", (rows, H)), cu_q=_ints(_starts(new)),
             conv_w=_rand(seed, "cw", (xbc, TAPS), -0.5, 0.5), conv_b=_randn(seed, "cb", (xbc,), std=0.02), A_log=_rand(seed, "A", (H,), 0.0, 2.0),
             Dskip=1.0 + _randn(seed, "D", (H,), std=0.1))
    step = torch.exp(_rand(seed, "bias", (H,), math.log(1e-3), math.log(1e-1)).double())
    s["dt_bias"] = (step + torch.log(-torch.expm1(-step))).float()                 # softplus of it is the step
    slots = B + 2
    s["slots"] = torch.randperm(slots, generator=_gen(seed, "slots"), device="cuda")[:B].to(torch.int32)
    s["conv"] = _randn(seed, "conv", (slots, TAPS - 1, xbc), kind)
    s["ssm"] = _randn(seed, "ssm", (slots, H, P, N), std=0.3)
    s["fresh"] = None if case["fresh"] == "none" else _ints(_fresh_of(case))
    s["keep"], s["keep_more"] = None, 0
    if case["mode"] == "look":
        s["keep"] = _ints(_kept_of(case))
    elif case["mode"] == "commit":                                                 # the drafts that stand, as a verification counts them
        s["keep"], s["keep_more"] = _ints([n - 1 for n in _kept_of(case)]), 1
    s["y"] = None if case["mode"] == "commit" else torch.zeros((rows, Di), dtype=KINDS[case["out"]], device="cuda")
    if own:                                                        # the scratch that the caller of this library owns
        import paper_2609_24197_b200 as hs
        s["workspace"] = torch.empty(hs.hspec_chunk_scan_workspace_bytes(rows, B, Di, P, N, G), dtype=torch.uint8, device="cuda")
    return s


def _prepare_logits(case, seed):
    B, V, new = case["batch"], case["vocab"], _rows_of(case)
    T = sum(new)
    rows, block = T + case["pad"], max(new)
    # logits as a language model has them: a wide bulk, and a few tokens far above it
    z = _randn(seed, "z", (rows, V), std=2.0)
    top = torch.randint(0, V, (rows, 6), generator=_gen(seed, "top"), device="cuda")
    z.scatter_(1, top, 9.0 + 7.0 * _rand(seed, "lead", (rows, 6)))
    s = dict(case=case, new=new, z=z.to(KINDS[case["kind"]]), cu_q=_ints(_starts(new)))
    s["out"] = s["z"] if case["place"] == "same" else torch.zeros((rows, V), dtype=KINDS[case["out"]], device="cuda")
    s["repetition"] = s["frequency"] = s["presence"] = s["history"] = s["bias_ids"] = s["mask"] = None
    if case["penalties"]:
        length = _spread(B, case["history_low"], case["history_high"])
        # words come back: half of a text's tokens are among its few most frequent
        wide = max(length) + 5
        common = (V * _rand(seed, "often", (B, wide)) ** 6).long().clamp(max=V - 1)
        rare = torch.randint(0, V, (B, wide), generator=_gen(seed, "rare"), device="cuda")
        s["history"] = torch.where(_rand(seed, "which", (B, wide)) < 0.5, common, rare).to(torch.int32)
        s["history_lens"], s["prompt_lens"] = _ints(length), _ints([n // 3 for n in length])
        s["drafts"] = torch.where(_rand(seed, "again", (B, block)) < 0.5, s["history"][:, :1], rare[:, :block] if wide >= block else rare[:, :1]).to(torch.int32)
        s["repetition"] = _rand(seed, "r", (B,), 0.9, 1.4)
        s["frequency"] = _rand(seed, "f", (B,), -0.2, 0.5)
        s["presence"] = _rand(seed, "p", (B,), -0.2, 0.8)
    if case["biases"]:
        n = case["biases"]
        s["bias_ids"] = torch.stack([torch.randperm(V, generator=_gen(seed, "bias%d" % b), device="cuda")[:n] for b in range(B)]).to(torch.int32)
        s["bias_values"] = _randn(seed, "bias", (B, min(n, V)), std=3.0)
        s["bias_counts"] = _ints([min(n, V) * (b + 1) // B for b in range(B)])
    if case["grammar"] != "none":
        # a grammar's state allows nearly all tokens (inside a string), or a few of them; a row of bits for every state that the rows are in
        words = -(-V // 32)
        any_ = torch.randint(-2**31, 2**31, (T, words), generator=_gen(seed, "any"), device="cuda")
        few = any_ & torch.randint(-2**31, 2**31, (T, words), generator=_gen(seed, "few"), device="cuda")
        few &= torch.randint(-2**31, 2**31, (T, words), generator=_gen(seed, "fewer"), device="cuda")
        open_ = any_ | few | torch.randint(-2**31, 2**31, (T, words), generator=_gen(seed, "more"), device="cuda")
        t = torch.arange(T, device="cuda")
        s["mask"] = torch.where((t % 2 == 0).unsqueeze(1), open_, few).to(torch.int32)
        rule = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        order = torch.randperm(T, generator=_gen(seed, "order"), device="cuda").to(torch.int32)
        rule[:T] = order if case["grammar"] == "all" else torch.where(t % 3 == 0, order, torch.full_like(order, -1))
        s["mask_rows"] = rule
    return s


def prepare(case, seed):
    return _prepare_scan(case, seed) if case["op"] == "scan" else _prepare_logits(case, seed)


# ------------------------------------------------------------------------------------------------ one pass

def _places(cu, rows):
    """Request of every row, and its index in that request's rows."""
    t = torch.arange(rows, device="cuda")
    b = torch.searchsorted(cu.long(), t, right=True) - 1
    return b, t - cu.long()[b]


def _plain_scan(s):
    """All requests at once, padded to one length, in chunks of Q rows: inside a chunk as a masked product, between chunks as a product with
    the chunks' decays."""
    case = s["case"]
    Di, P, N, G = SHAPES[case["shape"]]
    H, xbc, new, dev = Di // P, Di + 2 * G * N, s["new"], "cuda"
    B, T, most = len(new), sum(new), max(new)
    Q = min(64, most)
    C = -(-most // Q)
    slot = s["slots"].long()
    fresh = torch.zeros(B, device=dev) if s["fresh"] is None else s["fresh"].float()
    conv0 = s["conv"][slot].float() * (1 - fresh)[:, None, None]
    state0 = s["ssm"][slot] * (1 - fresh)[:, None, None, None]
    b, i = _places(s["cu_q"], T)
    count = (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    keep = count if s["keep"] is None else torch.minimum((s["keep"] + s["keep_more"]).long().clamp(min=0), count)

    # convolution over the carried rows and the new ones
    raw = torch.zeros((B, TAPS - 1 + C * Q, xbc), device=dev)
    raw[:, :TAPS - 1] = conv0
    raw[b, TAPS - 1 + i] = s["x"][:T, Di:Di + xbc].float()
    act = s["conv_b"].expand(B, C * Q, xbc).clone()
    act += raw[:, 0:C * Q] * s["conv_w"][:, 0]
    act += raw[:, 1:1 + C * Q] * s["conv_w"][:, 1]
    act += raw[:, 2:2 + C * Q] * s["conv_w"][:, 2]
    act += raw[:, 3:3 + C * Q] * s["conv_w"][:, 3]
    act = act / (1 + torch.exp(-act))
    tail = torch.gather(raw, 1, (keep.unsqueeze(1) + torch.arange(TAPS - 1, device=dev)).unsqueeze(2).expand(B, TAPS - 1, xbc))

    # steps; rows that are not kept add nothing to the state and do not let it decay
    v = (s["x"][:T, Di + xbc:].float() if s["dt"] is None else s["dt"][:T]) + s["dt_bias"]
    v = torch.where(v > 20, v, torch.log1p(torch.exp(v)))
    dt = torch.zeros((B, C * Q, H), device=dev)
    dt[b, i] = v
    rate = -torch.exp(s["A_log"].double())

    def chunks(t):
        return t.reshape(B, C, Q, *t.shape[2:])

    x, k, q = (chunks(t) for t in (act[..., :Di].reshape(B, C * Q, H, P), act[..., Di:Di + G * N].reshape(B, C * Q, G, N), act[..., Di + G * N:].reshape(B, C * Q, G, N)))

    def between(dt):
        """Products along chunks: what each chunk adds to the state, the decays' logarithms in 64 bits, and the state in front of every chunk."""
        fall = torch.cumsum(chunks(dt).double() * rate, 2)                                                    # [B, C, Q, H]
        weight = (torch.exp(fall[:, :, -1:] - fall).float() * chunks(dt)).permute(0, 1, 3, 2)                 # [B, C, H, Q]
        xw = (x.permute(0, 1, 3, 4, 2) * weight.unsqueeze(3)).reshape(B, C, G, H // G * P, Q)
        adds = torch.matmul(xw, k.permute(0, 1, 3, 2, 4)).reshape(B, C, H, P * N)
        adds = torch.cat([state0.reshape(B, 1, H, P * N), adds], 1)
        upto = torch.cumsum(torch.nn.functional.pad(fall[:, :, -1], (0, 0, 1, 0)), 1).permute(0, 2, 1)        # [B, H, C + 1]
        far = upto.unsqueeze(3) - upto.unsqueeze(2)
        later = torch.ones((C + 1, C + 1), dtype=torch.bool, device=dev).tril()
        far = torch.where(later, torch.exp(far.masked_fill(~later, 0.0)), 0.0).float()
        return fall, torch.matmul(far, adds.permute(0, 2, 1, 3))                                              # [B, H, C + 1, P N]

    if s["y"] is not None:
        fall, at = between(dt)
        near = fall.permute(0, 1, 3, 2).unsqueeze(4) - fall.permute(0, 1, 3, 2).unsqueeze(3)                  # [B, C, H, Q, Q]
        below = torch.ones((Q, Q), dtype=torch.bool, device=dev).tril()
        near = torch.where(below, torch.exp(near.masked_fill_(~below, 0.0)).float(), 0.0)
        score = torch.matmul(q.permute(0, 1, 3, 2, 4), k.permute(0, 1, 3, 4, 2))                              # [B, C, G, Q, Q]
        near = near.reshape(B, C, G, H // G, Q, Q) * score.unsqueeze(3) * chunks(dt).permute(0, 1, 3, 2).reshape(B, C, G, H // G, 1, Q)
        y = torch.matmul(near.reshape(B, C, H, Q, Q), x.permute(0, 1, 3, 2, 4))
        front = at[:, :, :-1].permute(0, 2, 1, 3).reshape(B, C, G, H // G * P, N)
        y0 = torch.matmul(q.permute(0, 1, 3, 2, 4), front.transpose(3, 4)).reshape(B, C, G, Q, H // G, P).permute(0, 1, 2, 4, 3, 5).reshape(B, C, H, Q, P)
        y += y0 * torch.exp(fall).float().permute(0, 1, 3, 2).unsqueeze(4)
        y = y.permute(0, 1, 3, 2, 4) + x * s["Dskip"][:, None]
        y = y.reshape(B, C * Q, Di)[b, i]
        z = s["x"][:T, :Di].float()
        s["y"][:T] = (y * (z / (1 + torch.exp(-z)))).to(s["y"].dtype)
    last = between(dt * (torch.arange(C * Q, device=dev) < keep.unsqueeze(1)).unsqueeze(2))[1][:, :, -1]
    changed = (keep > 0) | (fresh > 0)
    s["ssm"][slot[changed]] = last.reshape(B, H, P, N)[changed]
    s["conv"][slot[changed]] = tail[changed].to(s["conv"].dtype)
    return dict(ssm=s["ssm"], conv=s["conv"]) if s["y"] is None else dict(ssm=s["ssm"], conv=s["conv"], y=s["y"])


def _plain_logits(s):
    case = s["case"]
    B, V, T = case["batch"], case["vocab"], sum(s["new"])
    b, i = _places(s["cu_q"], T)
    z = s["z"][:T].to(torch.float32, copy=True)
    if s["history"] is not None:
        at = torch.arange(s["history"].shape[1], device="cuda")
        inside, mine = at < s["history_lens"].unsqueeze(1), at >= s["prompt_lens"].unsqueeze(1)
        ids = s["history"].long()
        said = torch.zeros((B, V), device="cuda").scatter_add_(1, ids, (inside & mine).float())
        prompt = torch.zeros((B, V), device="cuda").scatter_add_(1, ids, (inside & ~mine).float())
        n = said[b]
        before = torch.arange(s["drafts"].shape[1], device="cuda") < i.unsqueeze(1)
        n.scatter_add_(1, s["drafts"].long()[b], before.float())
        r = s["repetition"][b].unsqueeze(1)
        z = torch.where((n > 0) | (prompt[b] > 0), torch.where(z > 0, z / r, z * r), z)
        z -= s["frequency"][b].unsqueeze(1) * n
        z -= s["presence"][b].unsqueeze(1) * (n > 0)
    if s["bias_ids"] is not None:
        live = torch.arange(s["bias_ids"].shape[1], device="cuda") < s["bias_counts"].unsqueeze(1)
        z.scatter_add_(1, s["bias_ids"].long()[b], torch.where(live, s["bias_values"], 0.0)[b])
    if s["mask"] is not None:
        rule = s["mask_rows"][:T].long()
        bits = (s["mask"][rule.clamp(min=0)].unsqueeze(2) >> torch.arange(32, dtype=torch.int32, device="cuda")) & 1
        z.masked_fill_((bits.reshape(T, -1)[:, :V] == 0) & (rule >= 0).unsqueeze(1), float("-inf"))
    s["out"][:T] = z.to(s["out"].dtype)
    return s["out"]


def run(s):
    case = s["case"]
    if not own:
        return _plain_scan(s) if case["op"] == "scan" else _plain_logits(s)
    import paper_2609_24197_b200 as hs
    if case["op"] == "scan":
        hs.hspec_op_chunk_scan(s["x"], s["conv_w"], s["conv_b"], s["dt_bias"], s["A_log"], s["Dskip"], s["cu_q"], s["conv"], s["ssm"], s["y"],
                               s["workspace"], dt_raw=s["dt"], slots=s["slots"], fresh=s["fresh"], keep=s["keep"], keep_more=s["keep_more"])
        return dict(ssm=s["ssm"], conv=s["conv"]) if s["y"] is None else dict(ssm=s["ssm"], conv=s["conv"], y=s["y"])
    rules = {}
    if s["history"] is not None:
        rules.update(history=s["history"], history_lens=s["history_lens"], prompt_lens=s["prompt_lens"], drafts=s["drafts"], repetition=s["repetition"],
                     frequency=s["frequency"], presence=s["presence"])
    if s["bias_ids"] is not None:
        rules.update(bias_ids=s["bias_ids"], bias_values=s["bias_values"], bias_counts=s["bias_counts"])
    if s["mask"] is not None:
        rules.update(mask=s["mask"], mask_rows=s["mask_rows"])
    hs.hspec_op_adjust_logits(s["z"], s["out"], cu_q=s["cu_q"], **rules)
    return s["out"]


# ------------------------------------------------------------------------------------------------ accounting

def work(case):
    new = _rows_of(case)
    rows = float(sum(new))
    if case["op"] == "scan":
        Di, P, N, G = SHAPES[case["shape"]]
        H, xbc = Di // P, Di + 2 * G * N
        state, kept = 4.0 * Di * N + (TAPS - 1) * xbc * BYTES[case["kind"]], _kept_of(case)
        reads = sum(1 for f, n in zip(_fresh_of(case), kept) if not f and (n or case["mode"] != "commit"))
        writes = sum(1 for f, n in zip(_fresh_of(case), kept) if f or n)
        used = float(sum(kept)) if case["mode"] == "commit" else rows              # a commit needs no gate, and the accepted rows alone
        wide = (xbc + (0 if case["mode"] == "commit" else Di)) * BYTES[case["kind"]] + H * (BYTES[case["kind"]] if case["dt"] == "columns" else 4)
        out = 0 if case["mode"] == "commit" else Di * BYTES[case["out"]]
        each = (0.0 if case["mode"] == "commit" else 2.0) + (0.0 if case["mode"] == "look" else 3.0)
        return {"bytes": state * (reads + writes) + used * wide + rows * out, "flops": max(2.0, each) * used * Di * N}
    V = case["vocab"]
    masked = {"none": 0.0, "some": rows / 3, "all": rows}[case["grammar"]]
    if case["place"] == "same":                                    # what a rule forbids is written, a third or less of the words stay as they are
        return {"bytes": masked * (V / 8.0 + 0.5 * V * BYTES[case["kind"]]), "flops": masked * V}
    history = 4.0 * sum(_spread(case["batch"], case["history_low"], case["history_high"])) if case["penalties"] else 0.0
    return {"bytes": rows * V * (BYTES[case["kind"]] + BYTES[case["out"]]) + masked * V / 8.0 + history + 8.0 * case["batch"] * case["biases"],
            "flops": 2.0 * rows * V}


# ------------------------------------------------------------------------------------------------ by the definitions, in 64 bits

def _exact_scan(s):
    """Token by token: S <- exp(dt A) S + dt x B^T, y = S C + D x, times z's SiLU; requests side by side."""
    case = s["case"]
    Di, P, N, G = SHAPES[case["shape"]]
    H, xbc, new, cu = Di // P, Di + 2 * G * N, s["new"], s["cu_q"].tolist()
    fresh, kept, slot = _fresh_of(case), _kept_of(case), s["slots"].tolist()
    ssm, conv = s["ssm"].double(), s["conv"].double()
    y = None if s["y"] is None else s["y"].double()
    w, bias, A = s["conv_w"].double(), s["conv_b"].double(), -torch.exp(s["A_log"].double())
    S = torch.stack([torch.zeros_like(ssm[0]) if fresh[b] else ssm[slot[b]] for b in range(len(new))])
    rows = [torch.cat([torch.zeros_like(conv[0]) if fresh[b] else conv[slot[b]], s["x"][cu[b]:cu[b + 1], Di:Di + xbc].double()]) for b in range(len(new))]
    for b, n in enumerate(kept):
        if n or fresh[b]:
            conv[slot[b]] = rows[b][n:n + TAPS - 1]
            if n == 0:
                ssm[slot[b]] = 0.0
    for t in range(max(new)):
        here = [b for b in range(len(new)) if t < new[b]]
        line = torch.tensor([cu[b] + t for b in here], device="cuda")
        u = torch.stack([(rows[b][t:t + TAPS].T * w).sum(1) for b in here]) + bias
        u = u * torch.sigmoid(u)
        x, k, q = u[:, :Di].reshape(-1, H, P), u[:, Di:Di + G * N].reshape(-1, G, N), u[:, Di + G * N:].reshape(-1, G, N)
        k, q = (m.repeat_interleave(H // G, dim=1) for m in (k, q))
        raw = s["x"][line, Di + xbc:].double() if s["dt"] is None else s["dt"][line].double()
        dt = torch.logaddexp(raw + s["dt_bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        every = len(here) == len(new)
        Sh = S if every else S[here]
        Sh.mul_(torch.exp(dt * A)[:, :, None, None])
        Sh.add_((dt.unsqueeze(2) * x).unsqueeze(3) * k.unsqueeze(2))
        if not every:
            S[here] = Sh
        if y is not None:
            o = torch.matmul(Sh, q.unsqueeze(3)).squeeze(3) + s["Dskip"].double()[:, None] * x
            z = s["x"][line, :Di].double()
            y[line] = o.reshape(-1, Di) * z * torch.sigmoid(z)
        for j, b in enumerate(here):
            if kept[b] == t + 1:
                ssm[slot[b]] = Sh[j]
    return dict(ssm=ssm, conv=conv) if y is None else dict(ssm=ssm, conv=conv, y=y)


def _exact_logits(s):
    out, cu = s["out"].double(), s["cu_q"].tolist()
    V = s["case"]["vocab"]
    for b, n in enumerate(s["new"]):
        z = s["z"][cu[b]:cu[b + 1]].double()
        if s["history"] is not None:
            text, first = s["history"][b, :int(s["history_lens"][b])].long(), int(s["prompt_lens"][b])
            r, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
            for i in range(n):
                said = torch.bincount(torch.cat([text[first:], s["drafts"][b, :i].long()]), minlength=V)
                seen = (said > 0) | (torch.bincount(text[:first], minlength=V) > 0)
                row = torch.where(seen & (z[i] > 0), z[i] / r, torch.where(seen, z[i] * r, z[i]))
                z[i] = row - f * said.double() - p * (said > 0).double()
        if s["bias_ids"] is not None:
            m = int(s["bias_counts"][b])
            z[:, s["bias_ids"][b, :m].long()] += s["bias_values"][b, :m].double()
        for i in range(n):
            rule = -1 if s["mask"] is None else int(s["mask_rows"][cu[b] + i])
            if rule >= 0:
                v = torch.arange(V, device="cuda")
                z[i, (s["mask"][rule][v // 32] >> (v % 32).int()) % 2 == 0] = -math.inf
        out[cu[b]:cu[b + 1]] = z
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_scan(s) if case["op"] == "scan" else _exact_logits(s)
