"""GPU parity of the ragged chunk's operators (rotary positions and cache write, attention over the paged cache) against
oracle/target_oracle.py: odd sizes, mixed requests, masked places that hold NaN, bad pages, padded batches, captured calls."""
import numpy as np
import pytest
import torch

from oracle import target_oracle as to

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step, relative to the value


@pytest.fixture(scope="module")
def hs():
    import paper_2609_24197_b200 as m
    m.load_library()
    m.hspec_op_device_status(clear=True)
    return m


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(4711 + seed)


class Chunk:
    """A ragged chunk and its paged cache on the GPU.  Whatever no row may see is NaN: unused pages, places behind a request's last token,
    queries of padding rows."""

    def __init__(self, heads, dtype, new, past, page=16, pad=0, seed=0, spread=1.0, poison=True):
        self.Hq, self.Hkv, self.dh = heads
        self.dtype, self.page, self.new = dtype, page, list(new)
        g = _gen(seed)
        self.kv = [max(0, n + p) for n, p in zip(new, past)]           # (a negative past: more rows than cached tokens)
        self.B, self.rows = len(new), sum(new)
        cu = np.concatenate([[0], np.cumsum(new)])
        pages = [-(-c // page) for c in self.kv]
        perm = torch.randperm(sum(pages) + 3, generator=g).tolist()
        self.table = torch.full((self.B, max(1, max(pages))), -1, dtype=torch.int32)
        shape = (sum(pages) + 3, page, self.Hkv, self.dh)
        k, v = torch.randn(shape, generator=g), torch.randn(shape, generator=g)
        used = torch.zeros(shape[:2], dtype=torch.bool)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
            at += n
            for j in range(n):
                used[int(self.table[b, j]), :min(page, self.kv[b] - j * page)] = True
        if poison:
            k[~used], v[~used] = float("nan"), float("nan")
        self.k, self.v = k.to(dtype).cuda(), v.to(dtype).cuda()
        q = torch.randn((self.rows + pad, self.Hq, self.dh), generator=g) * spread
        q[self.rows:] = float("nan")
        self.q = q.to(dtype).cuda()
        self.cu, self.kv_lens, self.table = (torch.as_tensor(x, dtype=torch.int32).cuda() for x in (cu, self.kv, self.table))

    def run(self, hs, window=0, scale=0.0, q=None, o=None, ws=None, **other):
        q = self.q if q is None else q
        o = torch.full_like(self.q, 7.0) if o is None else o
        ws = self.workspace(hs) if ws is None else ws
        a = dict(k=self.k, v=self.v, table=self.table, cu=self.cu, kv=self.kv_lens)
        a.update(other)
        hs.hspec_op_chunk_attention(q, a["k"], a["v"], a["table"], a["cu"], a["kv"], o, ws, window=window, scale=scale)
        return o

    def workspace(self, hs):
        return torch.empty(hs.hspec_chunk_attention_workspace_bytes(self.Hq, self.Hkv, self.dh), dtype=torch.uint8, device="cuda")

    def reference(self, window=0, scale=None):
        """(o, the same with the values' absolute values) in 64 bits, request by request."""
        rep, out, size = self.Hq // self.Hkv, [], []
        cu, kv, table = self.cu.tolist(), self.kv_lens.tolist(), self.table.long()
        for b in range(self.B):
            n, L = cu[b + 1] - cu[b], kv[b]
            if n == 0:
                continue
            q = self.q[cu[b]:cu[b + 1]].double().reshape(n, self.Hkv, rep, self.dh).permute(1, 2, 0, 3)
            if L == 0:
                out.append(torch.zeros((n, self.Hq, self.dh), dtype=torch.float64, device="cuda"))
                size.append(out[-1])
                continue
            ids = table[b, :-(-L // self.page)]
            ok = ((ids >= 0) & (ids < self.k.shape[0]))
            K, V = (torch.where(ok[:, None, None, None], p[ids.clamp(0, self.k.shape[0] - 1)], 0).reshape(-1, self.Hkv, self.dh)[:L].double()
                    .permute(1, 0, 2) for p in (self.k, self.v))
            far = (torch.arange(L - n, L, device="cuda")[:, None] - torch.arange(L, device="cuda")[None])
            seen = (far >= 0) & ((far < window) if window else (far == far))
            z = torch.einsum("grnd,gjd->grnj", q, K) * (self.dh ** -0.5 if scale is None else scale)
            z = torch.where(seen, z, -torch.inf)
            e = torch.where(seen, torch.exp(z - z.amax(-1, keepdim=True)), 0.0)
            p = e / e.sum(-1, keepdim=True).clamp(min=1e-300)
            for x, to_ in ((V, out), (V.abs(), size)):
                to_.append(torch.einsum("grnj,gjd->ngrd", p, x).reshape(n, self.Hq, self.dh))
        z = torch.zeros((0, self.Hq, self.dh), dtype=torch.float64, device="cuda")
        return torch.cat(out + [z]), torch.cat(size + [z])

    def check(self, o, window=0, scale=None, what=""):
        """Every value within the roundings of the result (half a step of |o|) and of the softmax weights (half a step each, so half a step of
        sum p |v|); 2^-13 of the latter for exponentials and 32-bit sums.  fp16 weights under 2^-14 of the row's largest are off by up to 2^-25 of
        it: once more per key for values up to 6."""
        ref, size = self.reference(window, scale)
        h = HALF[self.dtype]
        bound = h * ref.abs() + (h + 2.0 ** -13) * size + (max(self.kv + [1]) * 2.0 ** -25 * 6 if self.dtype == torch.float16 else 0.0) + 1e-30
        got = o[:self.rows].double()
        assert torch.isfinite(got).all(), f"{what}: not finite"
        worst = ((got - ref).abs() / bound).max().item() if got.numel() else 0.0
        assert worst <= 1.0, f"{what}: {worst:.2f} times the bound"
        assert (o[self.rows:] == 7.0).all(), f"{what}: a padding row was written"
        return worst


HEADS = {"8b": (32, 8, 128), "32b": (64, 8, 128), "tiny": (4, 2, 64), "mha64": (3, 3, 64), "mqa": (24, 1, 128), "three": (6, 2, 128)}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads", sorted(HEADS))
def test_attention_of_mixed_requests(hs, heads, dtype):
    # single tokens, blocks, a prompt's piece, a request without rows, one without an earlier token, lengths around the tile sizes
    new, past = [1, 17, 0, 70, 1, 5, 33, 1, 128, 2], [0, 300, 40, 0, 127, 128, 1000, 129, 250, 2500]
    c = Chunk(HEADS[heads], dtype, new, past, seed=len(heads), pad=3)
    c.check(c.run(hs), what=heads)


@pytest.mark.parametrize("page", [1, 3, 8, 16, 24, 64, 128, 256])
@pytest.mark.parametrize("heads", ["three", "tiny"])
def test_attention_page_sizes(hs, heads, page):
    c = Chunk(HEADS[heads], torch.bfloat16, [1, 40, 7, 1], [700, 90, 0, 5], page=page, seed=page)
    c.check(c.run(hs), what=f"page {page}")


@pytest.mark.parametrize("window", [1, 7, 16, 128, 129, 1000, 100000])
@pytest.mark.parametrize("heads", ["8b", "mha64"])
def test_attention_windows(hs, heads, window):
    c = Chunk(HEADS[heads], torch.float16, [1, 17, 200, 1, 64], [3000, 1100, 77, 0, 300], page=8, seed=window)
    for b in range(c.B):                                    # pages that no row of the request sees may be gone
        first = max(0, c.kv[b] - c.new[b] - window + 1) // c.page
        c.k[c.table[b, :first].long()] = float("nan")
        c.v[c.table[b, :first].long()] = float("nan")
        c.table[b, :first] = -1
    o = c.run(hs, window=window)
    c.k, c.v = torch.nan_to_num(c.k), torch.nan_to_num(c.v)
    c.check(o, window=window, what=f"window {window}")
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


@pytest.mark.parametrize("heads,new,past", [("8b", [1], [20000]), ("8b", [17], [9000]), ("32b", [600], [3000]), ("mha64", [1000], [0]),
                                            ("8b", [1] * 40, list(range(1, 2001, 50))), ("32b", [16, 17, 32, 33] * 5, [64 * i for i in range(20)])])
def test_attention_long_and_wide(hs, heads, new, past):
    c = Chunk(HEADS[heads], torch.bfloat16, new, past, seed=len(new))
    c.check(c.run(hs), what=f"{heads} {len(new)}")


@pytest.mark.parametrize("heads", [(5, 5, 64), (14, 7, 128), (32, 16, 64), (32, 32, 128), (37, 37, 64), (64, 64, 64), (512, 1, 64), (1024, 2, 128), (129, 1, 64)])
def test_attention_head_counts(hs, heads):
    # groups of KV heads of every kind (one head, all of them, a part), and up to 512 rows of a single token
    c = Chunk(heads, torch.bfloat16, [3, 1, 0, 40], [500, 131, 7, 90], seed=heads[0])
    c.check(c.run(hs), what=str(heads))


FEW = {"8b": (32, 8, 128), "32b": (64, 8, 128), "mha64": (3, 3, 64), "tiny": (4, 2, 64), "seven": (35, 5, 128), "wide64": (128, 16, 64)}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads", sorted(FEW))
def test_attention_of_few_rows(hs, heads, dtype):
    # single tokens, some twos and threes, empty requests and one without an earlier token; lengths around the tiles and steps; one longer block
    rep = FEW[heads][0] // FEW[heads][1]
    most = max(1, 8 // rep)
    new = [1, 1, 0, min(2, most), 1, 1, most, 1, 0, 1, 1, 1, min(3, most), 1, 1]
    past = [0, 15, 3, 16, 62, 63, 64, 65, 9, 127, 128, 1000, 700, 5, 4095]
    for extra in ([], [8 // rep + 1]):
        c = Chunk(FEW[heads], dtype, new + extra, past + [333] * len(extra), seed=len(heads))
        c.check(c.run(hs), what=heads)


@pytest.mark.parametrize("page", [1, 3, 16, 24, 128])
@pytest.mark.parametrize("window", [0, 1, 17, 100, 2 ** 31 - 1])
def test_windows_and_pages_of_few_rows(hs, page, window):
    c = Chunk((4, 4, 128) if page % 2 else (16, 4, 64), torch.bfloat16, [1, 2, 1, 1, 2, 1], [500, 99, 0, 77, 1, 2000], page=page, seed=page)
    c.check(c.run(hs, window=window), window=window, what=f"page {page} window {window}")


def test_few_rows_without_a_place(hs):
    c = Chunk((4, 4, 64), torch.bfloat16, [6, 2, 1, 0], [-2, -2, 40, 5], seed=5)
    hs.hspec_op_device_status(clear=True)
    o = c.run(hs)
    c.check(o, what="no place")
    assert (o[:2] == 0).all() and (o[6:8] == 0).all() and (o[2] != 0).any()
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 2


@pytest.mark.parametrize("what", ["value", "key"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_few_rows_do_not_see_never_reaches_them(hs, what, bad):
    """Four tokens of a request whose third has a bad key or value, and a window that leaves a bad place to the first row alone."""
    c = Chunk((4, 2, 128), torch.bfloat16, [4, 1], [150, 3], page=16, seed=9)
    good = c.run(hs, window=100).clone()
    pool = c.v if what == "value" else c.k
    for key in (152, 51):                                    # row i stands at 150 + i and sees 51 + i .. 150 + i
        pool[c.table[0, key // 16].long(), key % 16, 1, 7] = bad
    o = c.run(hs, window=100)
    assert torch.equal(o[1], good[1]) and torch.equal(o[4], good[4]) and torch.equal(o[:, :2], good[:, :2])
    for row in (0, 2, 3):
        if what == "value":
            x = o[row, 2:, 7]
            assert torch.isnan(x).all() if bad != bad else (x == bad).all()
            assert torch.equal(o[row, 2:, 8:], good[row, 2:, 8:])
        else:                                                # (an infinite key is a score of +-infinity, of either sign for a query)
            assert torch.isnan(o[row, 2:]).any() or bad == bad
    hs.hspec_op_device_status(clear=True)


@pytest.mark.parametrize("spread", [0.0, 8.0, 40.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_flat_and_peaked_rows(hs, spread, dtype):
    c = Chunk(HEADS["8b"], dtype, [1] * 9, [3000, 64, 17, 900, 1, 0, 5000, 128, 2], seed=3, spread=spread)
    c.check(c.run(hs), what=f"spread {spread}")


def test_few_rows_same_bits_on_streams_and_in_graphs(hs):
    c = Chunk(HEADS["8b"], torch.bfloat16, [1, 2, 1], [3000, 700, 60], seed=13)
    first = c.run(hs).clone()
    side, outs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for s in side:
        with torch.cuda.stream(s):
            outs.append(c.run(hs, o=torch.full_like(c.q, 7.0), ws=c.workspace(hs)))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    graph, o, ws = torch.cuda.CUDAGraph(), torch.full_like(c.q, 7.0), c.workspace(hs)
    with torch.cuda.graph(graph):
        c.run(hs, o=o, ws=ws)
    for _ in range(2):
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, first)
    c.kv_lens -= 1
    c.cu[3] = c.cu[2]
    o.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    c.rows, c.kv = 3, [x - 1 for x in c.kv]
    c.check(o, what="replay")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_of_thousands_of_requests(hs, dtype):
    # the most requests, two thirds of them without a row: every CTA goes through many short items
    new = [(0, 1, 0, 2, 0, 0)[b % 6] for b in range(8192)]
    past = [(b * 37) % 150 for b in range(8192)]
    c = Chunk(HEADS["tiny"], dtype, new, past, seed=21)
    c.check(c.run(hs), what="many")


def test_attention_past_32_bit_offsets(hs):
    """Pools of more than 2^32 bytes with the request's pages at their ends, and rows of q and o that lie 2^27 values apart."""
    small = Chunk(HEADS["8b"], torch.bfloat16, [17, 1], [300, 900], seed=22, poison=False)
    want = small.run(hs)
    pages = 2 ** 32 // (16 * 8 * 128 * 2) + 500
    k, v = (torch.empty((pages, 16, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    n = small.k.shape[0]
    order = torch.randperm(n, generator=_gen(1))
    to_page = torch.where(order % 2 == 0, pages - 1 - order, order).cuda()
    k[to_page], v[to_page] = small.k, small.v
    table = torch.where(small.table >= 0, to_page[small.table.clamp(min=0).long()].to(torch.int32), -1).to(torch.int32)
    q, o = (torch.empty((17, 2 ** 27), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cut = small.cu.clone()
    cut[2] = 17                                              # (the second request's row does not fit: it has none)
    q[:, :4096], o[:, 4096] = small.q[:17].reshape(17, -1), 7.0
    small.run(hs, q=q[:, :4096].unflatten(1, (32, 128)), o=o[:, :4096].unflatten(1, (32, 128)), k=k, v=v, table=table, cu=cut)
    torch.cuda.synchronize()
    assert torch.equal(o[:, :4096].reshape(17, 32, 128), want[:17]) and (o[:, 4096] == 7.0).all()


def test_requests_that_share_pages(hs):
    """Two requests over the same prefix, and one whose cache names one page twice: read only, so they may."""
    c = Chunk(HEADS["three"], torch.bfloat16, [4, 9, 1], [60, 60, 63], seed=23)
    c.table[1, :3] = c.table[0, :3]
    c.table[2, 1] = c.table[2, 0]
    c.check(c.run(hs), what="shared")


@pytest.mark.parametrize("spread", [0.0, 8.0, 40.0])
def test_attention_of_flat_and_peaked_rows(hs, spread):
    # (scores up to some hundreds: the running maximum moves)
    c = Chunk(HEADS["8b"], torch.bfloat16, [1, 50, 130], [900, 400, 200], seed=3, spread=spread)
    for b, (n, L) in enumerate(zip(c.new, c.kv)):           # keys grow along the request, so that later ones outdo earlier ones
        for j in range(L):
            c.k[int(c.table[b, j // c.page]), j % c.page] *= 0.2 + 2.0 * j / L
    c.check(c.run(hs), what=f"spread {spread}")


def test_attention_scale(hs):
    c = Chunk(HEADS["three"], torch.float16, [3, 20], [50, 300], seed=9)
    c.check(c.run(hs, scale=0.03), scale=float(np.float32(0.03)), what="scale")


def test_rows_with_no_place_see_nothing(hs):
    c = Chunk(HEADS["three"], torch.bfloat16, [10, 200, 4], [-3, -150, -4], seed=5)       # 3 rows, 150 rows, all four of them
    hs.hspec_op_device_status(clear=True)
    o = c.run(hs)
    c.check(o, what="no place")
    assert (o[:3] == 0).all() and (o[10:160] == 0).all() and (o[210:] == 0).all() and (o[3] != 0).any()
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 3


@pytest.mark.parametrize("window", [1, 100, 2 ** 31 - 1])
def test_windows_of_rows_with_no_place(hs, window):
    """The largest window reaches back from a negative position past 32 bits."""
    c = Chunk(HEADS["8b"], torch.bfloat16, [10, 200, 4, 70], [-9, -150, -4, 300], seed=6)
    c.check(c.run(hs, window=window), window=window, what="no place")
    hs.hspec_op_device_status(clear=True)


@pytest.mark.parametrize("what", ["value", "key"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_never_reaches_it(hs, what, bad):
    """A token of the chunk whose key or value is not finite reaches itself and the rows behind it, no row in front of it."""
    c = Chunk(HEADS["8b"], torch.bfloat16, [60, 300], [90, 0], seed=6)
    clean = c.run(hs).clone()
    for b, j in ((0, 120), (1, 137), (1, 290)):
        (c.v if what == "value" else c.k)[int(c.table[b, j // 16]), j % 16, 1, 5] = bad
    o = c.run(hs)
    g = slice(4, 8)                                          # query heads of KV head 1
    assert torch.equal(o[:, :4], clean[:, :4]) and torch.equal(o[:, 8:], clean[:, 8:])
    for rows in (slice(0, 30), slice(60, 197)):
        assert torch.equal(o[rows, g], clean[rows, g])
    if what == "value":
        d = [i for i in range(128) if i != 5]
        for rows in (slice(30, 60), slice(197, 360)):
            assert torch.equal(o[rows, g][..., d], clean[rows, g][..., d])
            assert not torch.isfinite(o[rows, g, 5].float()).any()
        if bad == bad:
            assert (o[30:60, g, 5].float() == bad).all()


def test_row_pitch(hs):
    c = Chunk(HEADS["three"], torch.bfloat16, [1, 30], [100, 20], seed=8)
    wide = torch.full((c.rows, 3, 6, 128), float("nan"), dtype=c.dtype, device="cuda")
    wide[:, 1] = c.q
    out = torch.full((c.rows, 2, 6, 128), 7.0, dtype=c.dtype, device="cuda")
    c.run(hs, q=wide[:, 1], o=out[:, 1])
    c.check(out[:, 1], what="pitch")
    assert (out[:, 0] == 7.0).all()


def test_bad_pages_read_as_zeros_and_are_counted(hs):
    c = Chunk(HEADS["8b"], torch.bfloat16, [1, 20, 1], [600, 700, 40], seed=11)
    clean = c.run(hs).clone()
    hs.hspec_op_device_status(clear=True)
    c.table[0, 3], c.table[1, 40] = -5, c.k.shape[0] + 100
    o = c.run(hs)
    c.check(o, what="bad pages")
    assert torch.equal(o[21], clean[21])
    st = hs.hspec_op_device_status(clear=True)
    assert st["bad_inputs"] >= 2 and st["device_status"] == 0


def test_lengths_outside_are_held_and_counted(hs):
    c = Chunk(HEADS["three"], torch.bfloat16, [2, 3], [100, 30], seed=12)
    good = c.run(hs).clone()
    kv = c.kv_lens.clone()
    kv[1] = -7
    o = c.run(hs, kv=kv)
    assert torch.equal(o[:2], good[:2]) and (o[2:] == 0).all()
    kv[1] = 10 ** 9                                          # more than the page-table row holds: its end, through entries that name no page
    o = c.run(hs, kv=kv)
    assert torch.equal(o[:2], good[:2])                      # (the others now see the NaN behind the request's true end)
    cu = c.cu.clone()
    cu[2] = 10 ** 6                                          # more rows than the chunk has
    o = c.run(hs, cu=cu)
    assert torch.equal(o, good)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] > 0


def test_attention_same_bits_on_streams_and_in_graphs(hs):
    c = Chunk(HEADS["8b"], torch.bfloat16, [1, 17, 200], [3000, 700, 60], seed=13)
    first = c.run(hs).clone()
    side, outs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for s in side:                                           # two calls that may overlap, each with its own scratch
        with torch.cuda.stream(s):
            outs.append(c.run(hs, o=torch.full_like(c.q, 7.0), ws=c.workspace(hs)))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    graph, o, ws = torch.cuda.CUDAGraph(), torch.full_like(c.q, 7.0), c.workspace(hs)
    with torch.cuda.graph(graph):
        c.run(hs, o=o, ws=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, first)
    # the replay follows the arrays: one token less everywhere, and the last request without rows
    c.kv_lens -= 1
    c.cu[3] = c.cu[2]
    o.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    c.rows, c.kv = 18, [x - 1 for x in c.kv]
    c.check(o, what="replay")


# --------------------------------------------------------------------------- rotary positions and the cache write

def _rope_case(hs, heads, source, dtype, new, past, axes, layout=None, norm=True, page=16, pad=0, seed=0, base=0, gap=0, pos=True):
    Hq, Hkv, dh = HEADS[heads]
    c = Chunk(HEADS[heads], dtype, new, past, page=page, pad=pad, seed=seed, poison=False)
    g = _gen(seed + 1)
    T, width = c.rows + pad, (Hq + 2 * Hkv) * dh
    wide = torch.randn((T, width + gap), generator=g).to(source).cuda()
    qkv = wide[:, gap:] if gap else wide
    layout = [j % axes for j in range(dh // 2)] if layout is None else layout
    p = torch.randint(0, 5000, (axes, T), generator=g, dtype=torch.int32) + base
    qw, kw = (1.0 + 0.2 * torch.randn(dh, generator=g) for _ in range(2))
    before_k, before_v = c.k.clone(), c.v.clone()
    q = torch.full((T, Hq, dh), 7.0, dtype=dtype, device="cuda")
    hs.hspec_op_chunk_rope_write(qkv, p.cuda() if pos else None, layout if pos else None, c.cu, c.kv_lens, c.table, q, c.k, c.v, 1.0e6,
                                 q_norm_w=qw.cuda() if norm else None, k_norm_w=kw.cuda() if norm else None, eps=1e-6)
    torch.cuda.synchronize()
    x = qkv[:c.rows].double().cpu().numpy().reshape(c.rows, Hq + 2 * Hkv, dh)
    places = to.chunk_places(c.cu.tolist(), c.kv_lens.tolist())
    where = p[:, :c.rows].numpy() if pos else np.array([[at for _, at in places]])
    lay = layout if pos else [0] * (dh // 2)
    rq = to.chunk_rope(x[:, :Hq], where, lay, 1.0e6, qw.numpy() if norm else None)
    rk = to.chunk_rope(x[:, Hq:Hq + Hkv], where, lay, 1.0e6, kw.numpy() if norm else None)

    def close(got, ref, what, turned):
        # half a step of the result; angles off by 2^-22 (remainder and sincosf), the 32-bit norm and products by as much again, each a share
        # of the pair's length
        got, pairs = got.double().cpu().numpy(), len(lay)
        length = np.abs(ref)
        if turned:
            a, b = ref[..., :pairs], ref[..., pairs:2 * pairs]
            length = ref.copy()
            length[..., :pairs] = length[..., pairs:2 * pairs] = np.sqrt(a * a + b * b)
        bound = HALF[dtype] * np.abs(ref) + 2.0 ** -20 * np.abs(length) + 2.0 ** -25      # (fp16's smallest step)
        worst = np.max(np.abs(got - ref) / bound) if ref.size else 0.0
        assert worst <= 1.0, f"{what}: {worst:.2f} times the bound"

    close(q[:c.rows], rq, "queries", True)
    assert (q[c.rows:] == 7.0).all()
    table, touched = c.table.cpu().numpy(), torch.zeros(c.k.shape[:2], dtype=torch.bool)
    slots = [(int(table[b, at // page]), at % page) for b, at in places]
    i, j = torch.tensor([s[0] for s in slots]), torch.tensor([s[1] for s in slots])
    touched[i, j] = True
    close(c.k[i.cuda(), j.cuda()], rk, "keys", True)
    close(c.v[i.cuda(), j.cuda()], x[:, Hq + Hkv:], "values", False)
    keep = ~touched.cuda()
    assert torch.equal(c.k[keep], before_k[keep]) and torch.equal(c.v[keep], before_v[keep])


@pytest.mark.parametrize("source", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,dtype", [("8b", torch.bfloat16), ("32b", torch.float16), ("tiny", torch.bfloat16), ("mha64", torch.float16), ("mqa", torch.bfloat16)])
def test_rope_types_and_heads(hs, heads, dtype, source):
    _rope_case(hs, heads, source, dtype, [1, 0, 17, 5, 130], [40, 3, 0, 333, 16], axes=3, seed=len(heads), pad=2)


@pytest.mark.parametrize("axes,layout", [(1, [0] * 64), (2, [0] * 40 + [1] * 24), (3, [0] * 16 + [1] * 24 + [2] * 24), (8, None), (1, [0] * 8),
                                         (3, [0, 1, 2, 2, 1, 0, 0, 1] * 3)])
def test_rope_axes_and_partial_rotation(hs, axes, layout):
    _rope_case(hs, "three", torch.bfloat16, torch.bfloat16, [3, 20], [7, 50], axes=axes, layout=layout, norm=len(layout or []) != 24, seed=axes)


@pytest.mark.parametrize("rows", [1, 2, 31, 600, 5000])
def test_rope_row_counts_and_cache_positions(hs, rows):
    _rope_case(hs, "tiny", torch.bfloat16, torch.float16, [rows, 1], [3, 0], axes=1, pos=False, norm=rows % 2 == 0, seed=rows, page=3 if rows < 100 else 64)


def test_rope_far_positions(hs):
    _rope_case(hs, "three", torch.float32, torch.float16, [40], [0], axes=2, base=2 ** 31 - 6000, seed=1)


@pytest.mark.parametrize("gap", [1, 4, 8])
def test_rope_rows_off_the_vector_boundaries(hs, gap):
    for source in (torch.float32, torch.bfloat16):
        _rope_case(hs, "three", source, torch.bfloat16, [9, 2], [0, 4], axes=3, gap=gap, seed=gap)


def test_rope_past_32_bit_offsets(hs):
    """Rows of qkv 2^27 values apart, and a page past 2^32 bytes of the pools."""
    pages = 2 ** 32 // (16 * 2 * 128 * 2) + 3
    qkv = torch.empty((33, 2 ** 27), dtype=torch.bfloat16, device="cuda")
    row = torch.randn((33, 10 * 128), device="cuda").to(torch.bfloat16)
    qkv[:, :1280] = row
    k, v, few_k, few_v = (torch.zeros((n, 16, 2, 128), dtype=torch.bfloat16, device="cuda") for n in (pages, pages, 4, 4))
    cu, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 33], [40]))
    q, few_q = (torch.empty((33, 6, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hs.hspec_op_chunk_rope_write(row, None, None, cu, kv, torch.tensor([[1, 0, 2]], dtype=torch.int32, device="cuda"), few_q, few_k, few_v, 1.0e4)
    far = torch.tensor([[pages - 2, 0, pages - 1]], dtype=torch.int32, device="cuda")
    hs.hspec_op_chunk_rope_write(qkv[:, :1280], None, None, cu, kv, far, q, k, v, 1.0e4)
    torch.cuda.synchronize()
    assert torch.equal(q, few_q)
    for a, b in ((k, few_k), (v, few_v)):
        assert torch.equal(a[far[0].long()], b[[1, 0, 2]]) and not a[1:pages - 2].any() and b[[0, 1, 2]].any()


def test_rope_rows_without_a_place(hs):
    """More rows than cached tokens, and page ids that name no page: queries are written, the cache is not."""
    Hq, Hkv, dh = HEADS["three"]
    c = Chunk(HEADS["three"], torch.bfloat16, [6, 4], [-2, 10], seed=2, poison=False)
    qkv = torch.randn((10, (Hq + 2 * Hkv) * dh), device="cuda")
    q = torch.full((10, Hq, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    table = c.table.clone()
    table[1, 0] = c.k.shape[0] + 9
    k, v = c.k.clone(), c.v.clone()
    hs.hspec_op_device_status(clear=True)
    hs.hspec_op_chunk_rope_write(qkv, None, None, c.cu, c.kv_lens, table, q, c.k, c.v, 1.0e4)
    torch.cuda.synchronize()
    changed = (c.k != k).flatten(1).any(1)
    assert changed.nonzero().flatten().tolist() == [int(table[0, 0])]
    assert torch.equal(c.v[int(table[0, 0]), 4:], v[int(table[0, 0]), 4:])
    assert (q != 7.0).any(-1).all()
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 1 + 4


def test_rope_rows_of_offsets_that_do_not_ascend(hs):
    """A row that the offsets give to no request has nothing written, least of all through the next request's page-table entries."""
    Hq, Hkv, dh = HEADS["three"]
    table = torch.arange(8, dtype=torch.int32, device="cuda")[:, None]              # one page per request, and entries behind the last request's
    cu = torch.tensor([0, 20, 3, 3, 1, 30], dtype=torch.int32, device="cuda")       # rows 3 .. 19 are counted to request 3, which has none
    kv = torch.full((5,), 16, dtype=torch.int32, device="cuda")
    k, v = (torch.full((8, 16, Hkv, dh), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.full((30, Hq, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    hs.hspec_op_chunk_rope_write(torch.randn((30, (Hq + 2 * Hkv) * dh), device="cuda"), None, None, cu, kv, table[:5], q, k, v, 1.0e4)
    torch.cuda.synchronize()
    assert (q[3:20] == 7.0).all()
    for pool in (k, v):                                      # (request 4's own rows, 20 .. 29, go to places 6 .. 15 of its page)
        assert (pool[4, :6] == 5.0).all() and (pool[5:] == 5.0).all() and (pool[4, 6:] != 5.0).any(-1).all()
    hs.hspec_op_device_status(clear=True)


def test_rope_fp16_range(hs):
    c = Chunk(HEADS["three"], torch.float16, [1], [0], seed=2, poison=False)
    qkv = torch.full((1, 10 * 128), 1.0e6, device="cuda")
    q = torch.empty((1, 6, 128), dtype=torch.float16, device="cuda")
    hs.hspec_op_device_status(clear=True)
    hs.hspec_op_chunk_rope_write(qkv, None, None, c.cu, c.kv_lens, c.table, q, c.k, c.v, 1.0e4)
    assert (q == 65504).all() and (c.v[int(c.table[0, 0]), 0] == 65504).all()
    assert hs.hspec_op_device_status(clear=True)["f16_range_events"] == 10 * 128


def test_rope_in_a_graph(hs):
    Hq, Hkv, dh = HEADS["8b"]
    c = Chunk(HEADS["8b"], torch.bfloat16, [17, 1], [100, 20], seed=4, poison=False)
    qkv = torch.randn((18, (Hq + 2 * Hkv) * dh), device="cuda", dtype=torch.bfloat16)
    pos = torch.randint(0, 1000, (3, 18), dtype=torch.int32, device="cuda")
    axes = bytes([0] * 16 + [1] * 24 + [2] * 24)
    args = lambda q, k, v: (qkv, pos, axes, c.cu, c.kv_lens, c.table, q, k, v, 1.0e6)
    want = [torch.empty((18, Hq, dh), dtype=torch.bfloat16, device="cuda"), c.k.clone(), c.v.clone()]
    hs.hspec_op_chunk_rope_write(*args(*want))
    got = [torch.empty_like(want[0]), c.k.clone(), c.v.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hspec_op_chunk_rope_write(*args(*got))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c.kv_lens += 1                                           # the cache has moved on by a token
    graph.replay()
    for p, w in zip(got[1:], want[1:]):
        assert torch.equal(p[int(c.table[0, 117 // 16]), 117 % 16], w[int(c.table[0, 116 // 16]), 116 % 16])


def test_rope_counts_requests_without_rows_too(hs):
    """Lengths outside of requests that have no row in this chunk: as the attention over the same arrays counts them."""
    Hq, Hkv, dh = HEADS["three"]
    c = Chunk(HEADS["three"], torch.bfloat16, [2, 0, 0, 3], [8, 9, 9, 0], seed=2, poison=False)
    kv = torch.tensor([10, -3, 10 ** 6, 1], dtype=torch.int32, device="cuda")       # a good one, two without rows, one with more rows than tokens
    q = torch.empty((5, Hq, dh), dtype=torch.bfloat16, device="cuda")
    hs.hspec_op_device_status(clear=True)
    hs.hspec_op_chunk_rope_write(torch.randn((5, (Hq + 2 * Hkv) * dh), device="cuda"), None, None, c.cu, kv, c.table, q, c.k, c.v, 1.0e4)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 3
    c.run(hs, kv=kv)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 3


def _one_score_above_all_others(heads, dtype, new, past, size, sign):
    """q . k is sign 32 size^2 + order size^2 / 4096 with a whole number of its own for every key: exact in 32 bits, and no two scores of a row less than some
    ten thousand apart, so that every row takes the value at its largest."""
    c = Chunk(HEADS[heads], dtype, new, past, seed=17, poison=False)
    order = torch.randperm(int(max(c.kv)), generator=_gen(5)).cuda()
    c.q.zero_()
    c.k.zero_()
    c.q[..., 8:40], c.q[..., 4:6] = sign * size, size
    for b in range(c.B):
        at = torch.arange(c.kv[b], device="cuda")
        page, at = c.table[b].long()[at // c.page], at % c.page
        c.k[page, at, :, 8:40] = size
        c.k[page, at, :, 4] = ((order[:c.kv[b]] // 64) * (size / 64.0)).to(dtype)[:, None]
        c.k[page, at, :, 5] = ((order[:c.kv[b]] % 64) * (size / 4096.0)).to(dtype)[:, None]
    return c


@pytest.mark.parametrize("size", [2.0 ** 17, 2.0 ** 50, 2.0 ** 60])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size_of_few_rows(hs, sign, size):
    """Scores of 7e10 to 5e36, all of one sign: far below zero is not the same as unseen."""
    c = _one_score_above_all_others("tiny", torch.bfloat16, [1, 1, 1], [150, 5, 2000], size, sign)
    c.check(c.run(hs), what=f"size {size} sign {sign}")


@pytest.mark.parametrize("dtype,size", [(torch.bfloat16, 2.0 ** 17), (torch.bfloat16, 2.0 ** 50), (torch.bfloat16, 2.0 ** 60), (torch.float16, 2.0 ** 15)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("new,past", [([40, 300, 1], [150, 20, 700]), ([100, 17], [0, 3000])])
@pytest.mark.parametrize("heads", ["tiny", "8b"])
def test_scores_of_any_size(hs, heads, new, past, sign, dtype, size):
    """Scores of 4e9 to 5e36, all of one sign: a score's exact product with the scale and the row's rounded maximum may be thousands apart."""
    c = _one_score_above_all_others(heads, dtype, new, past, size, sign)
    c.check(c.run(hs), what=f"size {size} sign {sign}")
