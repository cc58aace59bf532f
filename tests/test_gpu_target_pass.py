"""The target's side of an iteration run as it is used: rotary positions and cache write, attention over the cache, LM head, verification, all of it one
captured graph that is replayed while requests grow by what was accepted and one of them ends."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import target_oracle as to

pytestmark = pytest.mark.gpu

B, K, V, PAGE, HQ, HKV, DH = 3, 6, 257, 8, 6, 2, 64


@pytest.fixture(scope="module")
def hs():
    import paper_2609_24197_b200 as m
    m.load_library()
    m.hspec_op_device_status(clear=True)
    return m


def _wide(t):
    return t.double().cpu().numpy()


class Pass:
    """Arrays of one pass of up to `rows` rows over B requests, at fixed addresses."""

    def __init__(self, hs, model, cache, rows):
        self.hs, self.model, self.cache = hs, model, cache
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
        self.ids, self.cu, self.kv = i32(rows), i32(B + 1), i32(B)
        self.q = torch.zeros((rows, HQ, DH), dtype=torch.bfloat16, device="cuda")
        self.o, self.logits = torch.zeros_like(self.q), torch.zeros((rows, V), device="cuda")
        self.ws = torch.empty(hs.hspec_chunk_attention_workspace_bytes(HQ, HKV, DH), dtype=torch.uint8, device="cuda")

    def set(self, rows, kv):
        """Token ids of every request's rows, and the cached tokens with them."""
        flat = [t for r in rows for t in r]
        self.ids.zero_()
        self.ids[:len(flat)] = torch.tensor(flat, dtype=torch.int32, device="cuda")
        self.cu.copy_(torch.tensor(np.concatenate([[0], np.cumsum([len(r) for r in rows])]), dtype=torch.int32))
        self.kv.copy_(torch.tensor(kv, dtype=torch.int32))

    def attend(self):
        m, c = self.model, self.cache
        self.hs.hspec_op_chunk_rope_write(m["qkv"][self.ids.long()], None, None, self.cu, self.kv, c["table"], self.q, c["k"], c["v"], 1.0e4)
        self.hs.hspec_op_chunk_attention(self.q, c["k"], c["v"], c["table"], self.cu, self.kv, self.o, self.ws)

    def head(self):
        self.hs.hspec_op_gemm(self.o.reshape(-1, HQ * DH), self.model["head"], self.logits, splits=1)


def _cache(seed):
    g = torch.Generator().manual_seed(seed)
    pages = 24
    pool = lambda: torch.full((B * pages + 2, PAGE, HKV, DH), float("nan"), dtype=torch.bfloat16, device="cuda")
    table = torch.randperm(B * pages, generator=g).reshape(B, pages).to(torch.int32).cuda()
    return dict(k=pool(), v=pool(), table=table)


def _places(cache, b, n):
    at = torch.arange(n, device="cuda")
    return cache["table"][b, at // PAGE].long(), at % PAGE


def test_iterations_of_a_target(hs):
    g = torch.Generator().manual_seed(5)
    model = dict(qkv=torch.randn((V, (HQ + 2 * HKV) * DH), generator=g).to(torch.bfloat16).cuda(),
                 head=(torch.randn((V, HQ * DH), generator=g) * 0.05).to(torch.bfloat16).cuda())
    cache = _cache(1)
    prompts = [torch.randint(0, V, (n,), generator=g).tolist() for n in (5, 70, 1)]
    seq = [list(p) for p in prompts]
    first = Pass(hs, model, cache, 80)                       # all of the prompts but their last tokens; the third has no row
    first.set([s[:-1] for s in seq], [len(s) - 1 for s in seq])
    first.attend()

    step = Pass(hs, model, cache, B * (K + 1))
    draft_logits = torch.zeros((B, K, V), device="cuda")
    ids, alpha, u = torch.zeros((B, K), dtype=torch.int32, device="cuda"), torch.zeros((B, K), device="cuda"), torch.zeros(B, device="cuda")
    n, tokens = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, K + 1), dtype=torch.int32, device="cuda")
    ws = torch.empty(hs.hspec_verify_workspace_bytes(B, K), dtype=torch.uint8, device="cuda")
    temperature = torch.tensor([1.0, 0.7, 0.0], device="cuda")

    def iteration():
        step.attend()
        step.head()
        hs.hspec_op_verify(step.logits, draft_logits, ids, alpha, u, n, tokens, ws, cu_q=step.cu, temperature=temperature)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iteration()
    counts = []
    for it in range(9):
        done = [False, it >= 6, False]                       # the second request ends
        z = torch.randn((B, K, V), generator=g) * 0.3
        d = torch.stack([torch.multinomial(torch.softmax(z[b] / 0.7 if b == 1 else z[b], 1), 1, generator=g).squeeze(1) for b in range(B)])
        if it == 3:                                          # the greedy request's drafts are the target's own here, from a pass of their own
            probe, own = Pass(hs, model, cache, B * (K + 1)), [seq[2][-1]]
            for j in range(K):
                probe.set([[], [], own], [0, 0, len(seq[2]) + j])
                probe.attend()
                probe.head()
                own.append(int(probe.logits[j].argmax()))
            d[2] = torch.tensor(own[1:])
        draft_logits.copy_(z)
        ids.copy_(d.to(torch.int32))
        alpha.copy_(torch.rand((B, K), generator=g))
        u.copy_(torch.rand(B, generator=g))
        rows = [[] if done[b] else [seq[b][-1]] + d[b].tolist() for b in range(B)]
        kv = [0 if done[b] else len(seq[b]) + K for b in range(B)]
        step.set(rows, kv)
        step.o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want_n, want = to.verify(_wide(step.logits), _wide(draft_logits), *(x.cpu().numpy() for x in (ids, alpha, u, step.cu)),
                                 temperature=temperature.cpu().numpy())
        np.testing.assert_array_equal(n.cpu().numpy(), want_n)
        np.testing.assert_array_equal(tokens.cpu().numpy(), want)
        # what was attended to: the committed tokens and the drafts, whatever refused drafts of earlier iterations have left behind
        used, at = sum(len(r) for r in rows), 0
        assert (step.o[used:] == 7.0).all()
        for b, r in enumerate(rows):
            if not r:
                assert tokens[b].tolist() == [-1] * (K + 1)
                continue
            full = seq[b] + r[1:]
            x = model["qkv"][torch.tensor(full)].double().cpu().numpy().reshape(len(full), HQ + 2 * HKV, DH)
            turned = to.chunk_rope(x[:, :HQ + HKV], np.arange(len(full))[None], [0] * (DH // 2), 1.0e4)
            rep = HQ // HKV
            q = turned[-len(r):, :HQ].reshape(len(r), HKV, rep, DH)
            s = np.einsum("ngrd,jgd->ngrj", q, turned[:, HQ:]) / np.sqrt(DH)
            seen = np.arange(len(full))[None] <= np.arange(len(full) - len(r), len(full))[:, None]
            s = np.where(seen[:, None, None], s, -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            v = x[:, HQ + HKV:]
            ref, size = (np.einsum("ngrj,jgd->ngrd", p, w).reshape(len(r), HQ, DH) for w in (v, np.abs(v)))
            # queries and keys are rounded to bf16 on the way: a score is off by 2 (2^-8 + 2^-20) sum |q k| / sqrt(dh), and the weights by e to that
            off = 2.0 * (2.0 ** -8 + 2.0 ** -20) * np.max(np.einsum("ngrd,jgd->ngrj", np.abs(q), np.abs(turned[:, HQ:]))) / np.sqrt(DH)
            bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -13 + np.expm1(2.0 * off)) * size
            assert (np.abs(_wide(step.o[at:at + len(r)]) - ref) <= bound).all()
            at += len(r)
            got = [t for t in tokens[b].tolist() if t >= 0]
            assert len(got) == int(n[b]) + 1 and got[:-1] == d[b, :int(n[b])].tolist()
            seq[b] += got
            counts.append(int(n[b]))
            if b == 2 and it == 3:
                assert int(n[b]) == K
    assert 0 < np.mean(counts) < K
    # the cache is, to the bit, what one pass over the accepted tokens leaves
    again = _cache(1)
    last = Pass(hs, model, again, sum(len(s) for s in seq))
    last.set([s[:-1] for s in seq], [len(s) - 1 for s in seq])
    last.attend()
    torch.cuda.synchronize()
    for b in range(B):
        i, j = _places(again, b, len(seq[b]) - 1)
        for pool in ("k", "v"):
            assert torch.isfinite(again[pool][i, j]).all() and torch.equal(cache[pool][i, j], again[pool][i, j])
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


FIRST_CALL = """
import sys, torch
import paper_2609_24197_b200 as hs
i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
half = lambda *s: torch.randn(s, device="cuda").to(torch.bfloat16)
u8 = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
table = i32(0, 1, 2, 3)[None]
k, v, q = half(4, 8, 2, 64), half(4, 8, 2, 64), half(3, 6, 64)
if sys.argv[1] == "write":
    qkv, out = half(3, 640), [torch.zeros_like(q), k, v]
    call = lambda: hs.hspec_op_chunk_rope_write(qkv, None, None, i32_cu, i32_kv, table, *out, 1.0e4)
elif sys.argv[1] == "attend":
    out, ws = [torch.zeros_like(q)], u8(hs.hspec_chunk_attention_workspace_bytes(6, 2, 64))
    call = lambda: hs.hspec_op_chunk_attention(q, k, v, table, i32_cu, i32_kv, out[0], ws)
else:
    z, ids, alpha, u, ws = torch.randn((3, 40), device="cuda"), i32(1, 2)[None], torch.rand((1, 2), device="cuda"), torch.rand(1, device="cuda"), u8(hs.hspec_verify_workspace_bytes(1, 2))
    out = [i32(-9), i32(-9, -9, -9)[None]]
    call = lambda: hs.hspec_op_verify(z, None, ids, alpha, u, out[0], out[1], ws)
i32_cu, i32_kv = i32(0, 3), i32(20)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call()
graph.replay()
torch.cuda.synchronize()
got = [x.clone() for x in out]
call()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, out)) and any((x != 0).any() for x in got)
assert not any(hs.hspec_op_device_status().values()), hs.hspec_op_device_status()
"""


@pytest.mark.parametrize("what", ["write", "attend", "verify"])
def test_the_first_call_of_a_process_may_be_a_captured_one(what):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALL, what], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-1500:]
