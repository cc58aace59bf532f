"""GPU parity of the verification of drafted tokens against oracle/target_oracle.py: both answers are integers and have to be equal."""
import numpy as np
import pytest
import torch

from oracle import target_oracle as to

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hs():
    import paper_2609_24197_b200 as m
    m.load_library()
    m.hspec_op_device_status(clear=True)
    return m


def _wide(t):
    return None if t is None else t.double().cpu().numpy()


def _run(hs, target, draft, ids, alpha, u, cu_q=None, vocab_map=None, temperature=None, ws=None):
    B, k = ids.shape
    n = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    tok = torch.full((B, k + 1), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty(hs.hspec_verify_workspace_bytes(B, k), dtype=torch.uint8, device="cuda") if ws is None else ws
    hs.hspec_op_verify(target, draft, ids, alpha, u, n, tok, ws, cu_q=cu_q, vocab_map=vocab_map, temperature=temperature)
    return n, tok


def _check(hs, target, draft, ids, alpha, u, cu_q=None, vocab_map=None, temperature=None):
    target, draft, ids, alpha, u, cu_q, vocab_map, temperature = (None if x is None else x.cuda() for x in
                                                                    (target, draft, ids, alpha, u, cu_q, vocab_map, temperature))
    n, tok = _run(hs, target, draft, ids, alpha, u, cu_q, vocab_map, temperature)
    a = [None if x is None else x.cpu().numpy() for x in (ids, alpha, u, cu_q, vocab_map, temperature)]
    want_n, want = to.verify(_wide(target), _wide(draft), *a)
    np.testing.assert_array_equal(n.cpu().numpy(), want_n)
    np.testing.assert_array_equal(tok.cpu().numpy(), want)
    return want_n, want


def _case(B, k, V, kind, seed, pruned=0, draft=True, right=0.7, spread=3.0):
    g = torch.Generator().manual_seed(99 + seed)
    Vd = pruned or V
    zt, zd = torch.randn((B * (k + 1), V), generator=g) * spread, torch.randn((B, k, Vd), generator=g) * spread
    vmap = torch.sort(torch.randperm(V, generator=g)[:Vd])[0].to(torch.int32) if pruned else None
    rows = (torch.arange(B)[:, None] * (k + 1) + torch.arange(k)[None]).flatten()
    same = rows[torch.rand(B * k, generator=g) < right]
    b, i = same // (k + 1), same % (k + 1)
    cols = torch.arange(V) if vmap is None else vmap.long()
    zt[same[:, None], cols] = zd[b, i] + 0.05 * zt[same[:, None], cols]
    zd, zt = zd.to(kind), zt.to(kind)
    q = torch.softmax(zd.float().reshape(B * k, Vd), 1)
    ids = (torch.multinomial(q, 1, generator=g).squeeze(1) if draft else q.argmax(1)).reshape(B, k)
    ids = ids if vmap is None else vmap.long()[ids]
    return dict(target=zt, draft=zd if draft else None, ids=ids.to(torch.int32), alpha=torch.rand((B, k), generator=g), u=torch.rand(B, generator=g),
                vocab_map=vmap)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,k,V", [(1, 1, 1), (1, 1, 2), (3, 7, 1000), (1, 16, 32000), (5, 33, 4099), (70, 5, 513), (300, 4, 100), (2, 3, 152064), (9, 2, 128257)])
def test_sampled_drafts(hs, B, k, V, kind):
    n, _ = _check(hs, **_case(B, k, V, kind, B + V))
    if B * k > 100:
        assert 0 < n.mean() < k


@pytest.mark.parametrize("spread", [0.0, 0.3, 12.0])
@pytest.mark.parametrize("draft", [True, False])
def test_flat_and_peaked_vocabularies(hs, draft, spread):
    for seed in range(4):
        _check(hs, **_case(4, 3, 50000, torch.float32, seed, draft=draft, spread=spread, right=0.5))


@pytest.mark.parametrize("B,k,V", [(1, 16, 32000), (40, 8, 2000), (200, 16, 300)])
def test_argmax_drafts(hs, B, k, V):
    _check(hs, **_case(B, k, V, torch.float32, V, draft=False, right=0.9, spread=6.0))


@pytest.mark.parametrize("V,pruned", [(1000, 1), (1000, 37), (4099, 1000), (152064, 32000), (513, 513)])
def test_pruned_vocabulary(hs, V, pruned):
    for B, k in ((3, 5), (64, 2)):
        _check(hs, **_case(B, k, V, torch.bfloat16, V + B, pruned=pruned, right=0.4))


def test_temperatures_and_ragged_rows(hs):
    B, k, V = 24, 6, 3001
    for seed, pruned in ((0, 0), (1, 800)):
        c = _case(B, k, V, torch.float32, seed, pruned=pruned)
        c["temperature"] = torch.tensor([1.0, 0.0, 0.3, 2.5, 1e-6, 40.0] * 4)
        rows = torch.tensor([0, 1, 2, 5, 7, 7, 3, 9, 6, 7, 1, 4] * 2)                # none, a token alone, more than k + 1
        cu = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(rows, 0)]).to(torch.int32)
        assert int(cu[-1]) <= c["target"].shape[0]
        _check(hs, cu_q=cu, **c)


def test_greedy_ties_take_the_lowest(hs):
    V = 777
    z = torch.zeros((4, V))
    z[0, [5, 300, 776]] = 3.0
    z[2, [0, 776]] = 1.0
    ids = torch.tensor([[5], [0]], dtype=torch.int32)
    n, tok = _check(hs, z, None, ids, torch.tensor([[0.5], [0.5]]), torch.tensor([0.9, 0.9]), temperature=torch.zeros(2))
    assert n.tolist() == [1, 1] and tok.tolist() == [[5, 0], [0, 0]]


def test_masked_tokens_and_rows_without_weight(hs):
    V, inf = 500, float("inf")
    g = torch.Generator().manual_seed(1)
    z = torch.randn((8, V), generator=g)
    d = torch.randn((4, 1, V), generator=g)
    ids = torch.tensor([[3], [4], [5], [6]], dtype=torch.int32)
    z[0, 3] = -inf                                           # masked: never stands, at alpha 0 either
    z[2, 10:] = float("nan")
    z[4] = -inf                                              # nothing to take: token 0
    z[6, 6] = inf                                            # counts as the largest finite number: all of p
    d[1, 0, 4] = -inf                                        # q = 0 at a token with p > 0: stands
    d[2] = -inf
    for alpha in (0.0, 1e-38, 0.5, 1.0):
        _check(hs, z, d, ids, torch.full((4, 1), alpha), torch.tensor([0.0, 0.3, 0.7, 0.99999994]))
    _check(hs, z, d, ids, torch.full((4, 1), 0.5), torch.rand(4, generator=g), temperature=torch.tensor([0.0, 1.0, 0.0, 3.0]))


def test_probabilities_next_to_alpha(hs):
    """alpha at the ratio itself and one step of 32 bits to either side: the 64-bit comparison decides."""
    B, V = 96, 20011
    c = _case(B, 1, V, torch.float32, 5, right=0.0, spread=1.5)
    p, q = (torch.softmax(c[x].double().reshape(B, -1, V)[:, 0], 1) for x in ("target", "draft"))
    x = c["ids"].long()
    ratio = (p.gather(1, x) / q.gather(1, x)).float().clamp(max=1.0)
    step = torch.tensor([0.0, -1.0, 1.0] * 32)[:, None] * ratio * 2.0 ** -23
    c["alpha"] = (ratio + step).clamp(max=1.0)
    n, _ = _check(hs, **c)
    assert 0 < n.sum() < B


def test_uniform_numbers_next_to_a_cumulative_sum(hs):
    """u at the borders between tokens of a flat vocabulary (k / V is exact where V is a power of two, or next to it), and out of range."""
    V = 4096
    z = torch.zeros((16, V))
    u = torch.tensor([0.0, 1 / V, 2 / V, 0.5, 1 - 1 / V, 0.99999994, 1 / V - 2.0 ** -36, 1.0])
    ids = torch.zeros((8, 1), dtype=torch.int32)
    n, tok = _run(hs, z.cuda(), None, ids.cuda(), torch.full((8, 1), 0.0, device="cuda"), u.cuda())
    assert n.tolist() == [1] * 8 and tok[:, 1].tolist() == [0, 1, 2, V // 2, V - 1, V - 1, 0, V - 1]


def test_probabilities_that_64_bits_do_not_hold(hs):
    """A low temperature: p and q of the drafted token at 2^-900 .. 2^-1100, where they lose bits and become nothing, with their ratio near 1."""
    B, V = 64, 12
    z, d = torch.zeros((2 * B, V)), torch.zeros((B, 1, V))
    depth = torch.linspace(620.0, 765.0, B)                  # of the token, in units of the temperature (2^-1022 is e^-708, the least is e^-745)
    temperature = torch.full((B,), 2.0 ** -10)
    z[0::2, 3] = -depth * 2.0 ** -10
    d[:, 0, 3] = (-depth + torch.tensor([1.5, -1.5]).repeat(B // 2)) * 2.0 ** -10
    n, _ = _check(hs, z, d, torch.full((B, 1), 3, dtype=torch.int32), torch.full((B, 1), 0.5), torch.full((B,), 0.4), temperature=temperature)
    assert 0 < n.sum() < B // 2


@pytest.mark.parametrize("draft", [True, False])
def test_the_least_weights_at_u_zero(hs, draft):
    """u = 0 takes the lowest token with any weight in 64 bits: one of e^-650 .. e^-760 of the largest, in front of it."""
    B, V = 48, 600
    z, d = torch.full((2 * B, V), -1.0e30), torch.full((B, 1, V), -1.0e30)
    depth = torch.linspace(650.0, 760.0, B)
    z[:, 400] = d[:, 0, 500] = 0.0
    z[0::2, 7] = z[1::2, 7] = -depth * 2.0 ** -10
    ids = torch.full((B, 1), 500, dtype=torch.int32)
    for alpha in (0.5, 0.0):
        n, tok = _check(hs, z, d if draft else None, ids, torch.full((B, 1), alpha), torch.zeros(B), temperature=torch.full((B,), 2.0 ** -10))
        assert set(tok[:, 0].tolist()) == {7, 400}


def test_rows_that_agree_but_for_next_to_nothing(hs):
    """p and q have the same token at 1 to the bit, and differ in another at e^-600: that is all of max(0, p - q)."""
    B, V = 60, 103
    g = torch.Generator().manual_seed(4)
    top = torch.randint(0, 50, (B,), generator=g)
    m = torch.randn(B, generator=g) * 9.0
    z, d = (torch.full((B, V), -1.0e4) for _ in range(2))
    at = torch.arange(B)
    z[at, top] = d[at, top] = m
    z[at, 50 + top] = m - 0.6
    d[at, 102] = m - 0.5
    both = torch.stack([z, z], 1).reshape(2 * B, V)
    n, tok = _check(hs, both, d[:, None], torch.full((B, 1), 102, dtype=torch.int32), torch.full((B, 1), 0.9), torch.rand(B, generator=g),
                    temperature=torch.full((B,), 1e-3))
    assert n.sum() == 0 and tok[:, 0].tolist() == (50 + top).tolist()


def test_what_an_argmax_drafter_leaves_over(hs):
    """The refused token holds nearly all of p: the rest is as small as 2^-39 of it, and its tokens are alike or far apart."""
    B, V = 240, 5003
    g = torch.Generator().manual_seed(77)
    z = torch.randn((B, 2, V), generator=g)
    z[0::3] = 0.0
    z[1::3, :, 40:] = -float("inf")
    ids = torch.randint(0, 40, (B, 1), generator=g, dtype=torch.int32)
    gap = torch.linspace(4.0, 30.0, B)
    z[torch.arange(B), 0, ids[:, 0].long()] = gap + 1.0
    n, _ = _check(hs, z.reshape(2 * B, V), None, ids, torch.ones((B, 1)), torch.rand(B, generator=g))
    assert n.sum() == 0


def test_a_draft_outside_the_vocabulary_does_not_stand(hs):
    c = _case(3, 2, 900, torch.float32, 3)
    c["ids"][0, 0], c["ids"][1, 1] = -1, 900
    hs.hspec_op_device_status(clear=True)
    n, _ = _check(hs, **c)
    assert n[0] == 0 and n[1] <= 1
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] >= 1


def test_row_pitch_and_odd_addresses(hs):
    c = {k: v.cuda() if v is not None else None for k, v in _case(4, 3, 1001, torch.bfloat16, 8).items()}
    want = _run(hs, **c)
    wide = torch.full((16, 1007), float("nan"), dtype=torch.bfloat16, device="cuda")
    for first in (0, 1, 3, 6):
        wide[:, first:first + 1001] = c["target"]
        got = _run(hs, **dict(c, target=wide[:, first:first + 1001]))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_past_32_bit_offsets(hs):
    c = {k: v.cuda() if v is not None else None for k, v in _case(4, 4, 5001, torch.bfloat16, 12).items()}
    want = _run(hs, **c)
    far = torch.empty((20, 2 ** 27), dtype=torch.bfloat16, device="cuda")
    far[:, :5001] = c["target"]
    got = _run(hs, **{**c, "target": far[:, :5001]})
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_thousands_of_requests(hs):
    _check(hs, **_case(9000, 2, 33, torch.float16, 13))


def test_streams_and_graphs(hs):
    c = {k: v.cuda() if v is not None else None for k, v in _case(130, 12, 1500, torch.float32, 2).items()}
    want = [x.clone() for x in _run(hs, **c)]
    side, outs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for s in side:
        with torch.cuda.stream(s):
            outs.append(_run(hs, **c))
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(a, b) for a, b in zip(o, want))
    ws = torch.randint(0, 255, (hs.hspec_verify_workspace_bytes(130, 12),), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _run(hs, ws=ws, **c)
    for _ in range(3):
        ws.random_(0, 255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    c["alpha"].fill_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    again = _run(hs, **c)
    assert all(torch.equal(a, b) for a, b in zip(got, again)) and not torch.equal(got[0], want[0])


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
def test_no_draft_stands_on_a_row_without_weight(hs, kind):
    """Greedy requests whose draft's row is -infinity all through: token 0 is what comes out of it, but as the target's, not as a draft that stands."""
    V = 300
    z = torch.randn((8, V), generator=torch.Generator().manual_seed(7)).to(kind)
    z[0::2] = -float("inf")
    for warm in (0.0, 1.0):
        n, tok = _check(hs, z, None, torch.tensor([[0], [1], [0], [299]], dtype=torch.int32), torch.zeros((4, 1)), torch.full((4,), 0.5),
                        temperature=torch.full((4,), warm))
        assert n.tolist() == [0] * 4 and tok.tolist() == [[0, -1]] * 4


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
def test_nan_logits_lose_every_argmax(hs, kind):
    """Runs of NaN that fill whole 16-byte words, alone and beside +infinity, in the rows whose arg-max counts: a greedy request's draft rows, and the
    row behind drafts that all stand, of greedy and of sampling requests."""
    V, g = 1037, torch.Generator().manual_seed(31)          # (an odd pitch: words begin anywhere in a row)
    runs = [(0, 16), (0, 1), (7, 9), (256, 288), (500, 541), (V - 16, V), (V - 37, V), (1, V), (0, V - 1), (0, V)]
    top = [None, 0, 1, 5, 15]                               # place of a +infinity within the run
    z, ids, warm, alpha = [], [], [], []
    for first, end in runs:
        for inf in top:
            for how in range(4):
                rows = (torch.randn((2, V), generator=g) * 3.0).to(kind)
                drafted = int(rows[0].float().argmax())
                bad = rows[0] if how in (0, 3) else rows[1]
                bad[first:end] = float("nan")
                if inf is not None and first + inf < end:
                    bad[first + inf] = float("inf")
                if how == 0:                                # the row's arg-max, where it has one
                    drafted = int(torch.nan_to_num(bad.float(), nan=-float("inf"), posinf=3.4e38).argmax())
                z.append(rows)
                ids.append([drafted])
                warm.append(0.0 if how < 2 else 1.0)
                alpha.append([1.0 if how == 3 else 0.0])
    B = len(ids)
    n, tok = _check(hs, torch.cat(z), None, torch.tensor(ids, dtype=torch.int32), torch.tensor(alpha), torch.rand(B, generator=g),
                    temperature=torch.tensor(warm))
    assert (n[0::4][:-5] == 1).all() and (n[1::4] == 1).all()        # (the last five have nothing but NaN in the draft's row, or +infinity beside it)


@pytest.mark.parametrize("V", [50000, 152064])
@pytest.mark.parametrize("where", ["draft", "target"])
def test_deep_tokens_of_flat_rows(hs, where, V):
    """Tokens some 700 temperatures below thousands of equal ones: next to nothing of a sum of V, which a 64-bit exponent holds only with care.  In the draft's
    row they must not take the rest; in the target's, in front of all others, u = 0 takes the first of them that has any weight at all."""
    depth = torch.arange(640.0, 725.0, 0.25)
    z, d = torch.zeros((8, V)), torch.zeros((4, 1, V))
    z[0::2, V - 20:] = 0.5                                  # what is left of p - q, and next to none of it: decided in 64 bits
    if where == "draft":
        z[0::2, 100:100 + depth.numel()] = d[:, 0, 100:100 + depth.numel()] = -depth
        z[0::2, 100:100 + depth.numel()] -= 1.0
        u = torch.tensor([0.0, 0.3, 0.7, 0.999])
    else:
        for b in range(4):
            z[2 * b, 0] = -(697.0, 698.25, 699.0, 699.75)[b]
        d[:, 0, 0] = -1.0e30
        u = torch.zeros(4)
    ids = torch.full((4, 1), V // 2, dtype=torch.int32)
    n, tok = _check(hs, z, d, ids, torch.ones((4, 1)), u)
    assert n.sum() == 0 and ((tok[:, 0] >= V - 20).all() if where == "draft" else (tok[:, 0] == 0).all())


@pytest.mark.parametrize("depth,side", [(2.8125, 1), (3.53125, -1)])
def test_the_accept_test_of_a_huge_vocabulary(hs, depth, side):
    """2^27 tokens, all but some of them `depth` below the largest: a running sum in 32 bits that comes by every 4096th word of an eighth of them is off by 2.9e-5
    here (the same rounding of every addition, down for one depth and up for the other), and alpha lies halfway between the drafted token's share and what such a
    sum makes of it."""
    V, tops = 2 ** 27, 2 ** 12
    p = np.exp(-depth) / (8 * tops + (V - 8 * tops) * np.exp(-depth))
    z = torch.full((2, V), -depth, dtype=torch.float16, device="cuda")
    z[0].view(8, -1)[:, :tops] = 0.0                         # (a running maximum that is there from the first word on)
    alpha = np.float32(p * (1.0 + side * 1.45e-5))
    assert (p >= float(alpha)) == (side < 0)
    n, tok = _run(hs, z, None, torch.full((1, 1), V - 1, dtype=torch.int32, device="cuda"), torch.full((1, 1), float(alpha), device="cuda"),
                  torch.zeros(1, device="cuda"))
    assert n.tolist() == [int(side < 0)] and tok.tolist() == [[V - 1, 0] if side < 0 else [0, -1]]


def test_offsets_far_outside_are_held(hs):
    """Entries of cu_q at the ends of 32 bits: a request that they give no row has none, and the others are as they were."""
    B, k, V = 5, 3, 50
    c = _case(B, k, V, torch.float32, 41)
    low, high = -2 ** 31, 2 ** 31 - 1
    c["target"] = c["target"][:2].clone()                   # (fewer rows than a request may have)
    for cu, rows in (([0, low, 2, 2, 2, 2], [0, 2, 0, 0, 0]), ([low, 1, high, 2, low, high], [1, 1, 0, 0, 2]), ([2, 2, high, high, 0, 1], [0, 0, 0, 0, 1]),
                     ([high, low, high, low, low, 2], [0, 2, 0, 0, 2])):
        offsets = torch.tensor(cu, dtype=torch.int32)
        n, tok = _run(hs, **{x: None if y is None else y.cuda() for x, y in dict(c, cu_q=offsets).items()})
        first = [min(max(x, 0), 2) for x in cu[:-1]]
        for b in range(B):
            one = to.verify(_wide(c["target"]), _wide(c["draft"][b:b + 1]), *(c[x][b:b + 1].numpy() for x in ("ids", "alpha", "u")),
                            cu_q=[first[b], first[b] + rows[b]])
            assert n[b].item() == one[0][0] and tok[b].tolist() == one[1][0].tolist(), (cu, b)
    hs.hspec_op_device_status(clear=True)


def test_the_rest_of_a_draft_that_no_ratio_reaches(hs):
    """alpha above 1 refuses whatever stands: an arg-max drafter's token may then hold all of p but weights that 32 bits flush to nothing, one by one or
    many of them beside a larger one."""
    B, V = 60, 50021
    g = torch.Generator().manual_seed(51)
    z = torch.full((B, 2, V), -float("inf"))
    at = torch.randint(0, V - 1, (B,), generator=g)
    for b in range(B):
        if b % 3 == 0:                                      # a few tokens, the largest at e^-80 .. e^-700
            z[b, :, torch.randint(0, V, (30,), generator=g)] = -torch.linspace(80.0, 700.0, B)[b] - 3.0 * torch.rand(30, generator=g)
        elif b % 3 == 1:                                    # all of them under 2^-126 = e^-87.3
            z[b] = -88.0 - 4.0 * torch.rand(V, generator=g)
        else:                                               # the same and one above it
            z[b] = -88.0 - 0.5 * torch.rand(V, generator=g)
            z[b, :, V - 1] = -87.0
        z[b, :, at[b]] = 0.0
    alpha = torch.full((B, 1), 2.0)
    alpha[1::7] = float("nan")
    n, tok = _check(hs, z.reshape(2 * B, V), None, at[:, None].to(torch.int32), alpha, torch.rand(B, generator=g))
    assert n.sum() == 0 and (tok[:, 0] != at.numpy()).all()


@pytest.mark.parametrize("V", [40, 30000])
def test_the_largest_and_the_smallest_temperatures(hs, V):
    """Temperatures up to 1e36 and down to 1e-36 count as they are, over logits of their size; those beyond count as 1e36 and 1e-36."""
    g = torch.Generator().manual_seed(61)
    T = [1e29, 1e30, 3e30, 1e33, 9e35, 1e36, 3e38, float("inf"), 1e-29, 1e-30, 3e-31, 1e-33, 2e-36, 1e-36, 1e-38, 1e-45]
    t = torch.tensor(T)
    held = t.clamp(1e-36, 1e36)
    B, k = len(T), 2
    z, d = (torch.randn((B, n, V), generator=g) * 2.0 * held[:, None, None] for n in (k + 1, k))
    z[:, 0] = d[:, 0] + 0.02 * z[:, 0]
    z[:8, :, 7] = -float("inf")                             # masked tokens stay masked
    z[:, :, 11] = -3.0e38
    c = dict(target=z.reshape(-1, V), draft=d, ids=torch.randint(12, V, (B, k), generator=g, dtype=torch.int32), alpha=torch.rand((B, k), generator=g),
             u=torch.rand(B, generator=g))
    n, tok = _run(hs, **{x: y.cuda() for x, y in c.items()}, temperature=t.cuda())
    want_n, want = to.verify(_wide(c["target"]), _wide(d), *(c[x].numpy() for x in ("ids", "alpha", "u")), temperature=held.numpy())
    np.testing.assert_array_equal(n.cpu().numpy(), want_n)
    np.testing.assert_array_equal(tok.cpu().numpy(), want)
    assert 0 < want_n.sum() < B * k


def test_offsets_outside_are_counted(hs):
    c = {x: None if y is None else y.cuda() for x, y in _case(6, 2, 60, torch.float32, 71).items()}
    hs.hspec_op_device_status(clear=True)
    _run(hs, **c)
    _run(hs, **dict(c, cu_q=torch.tensor([0, 3, 3, 4, 9, 12, 18], dtype=torch.int32, device="cuda")))
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0
    _run(hs, **dict(c, cu_q=torch.tensor([-1, 3, 2, 4, 9, 12, 19], dtype=torch.int32, device="cuda")))
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 3          # in front of the rows, descending, behind them


def test_an_iteration_in_which_no_request_has_rows(hs):
    c = {x: None if y is None else y.cuda() for x, y in _case(4, 3, 70, torch.bfloat16, 81).items()}
    for draft in (c["draft"], None):
        n, tok = _run(hs, **dict(c, target=c["target"][:0], draft=draft, cu_q=torch.zeros(5, dtype=torch.int32, device="cuda")))
        assert n.tolist() == [0] * 4 and tok.tolist() == [[-1] * 4] * 4
    with pytest.raises(hs.HSpecError, match="k \\+ 1 rows"):
        _run(hs, **dict(c, target=c["target"][:0]))


@pytest.mark.parametrize("draft", [True, False])
def test_greedy_drafts_that_no_ratio_reaches(hs, draft):
    """min(1, p / q) is 1 for a greedy request's arg-max: an alpha above that, or NaN, refuses it, and the target's token is the same."""
    c = _case(6, 3, 500, torch.float32, 91, draft=draft)
    c["ids"] = c["target"].reshape(6, 4, 500)[:, :3].argmax(-1).to(torch.int32)
    c["alpha"] = torch.tensor([[1.0, 1.0, 1.0], [1.0000001, 0.0, 0.0], [0.5, float("nan"), 0.5], [0.5, 0.5, 2.0], [-1.0, 0.0, 1.0], [float("inf"), 0.0, 0.0]])
    n, tok = _check(hs, **c, temperature=torch.zeros(6))
    assert n.tolist() == [3, 0, 1, 2, 3, 0]


@pytest.mark.parametrize("kinds", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("V,pitch", [(157, 160), (3001, 3001), (40009, 40013)])
def test_equal_rows_at_any_alignment(hs, V, pitch, kinds):
    """A drafter that is the target, its rows elsewhere in memory and of another type: every ratio is 1 to the bit, and nothing is left of p - q."""
    B, k, g = 9, 4, torch.Generator().manual_seed(V)
    d = (torch.randn((B, k, V), generator=g) * 2.0).to(torch.float16).to(torch.bfloat16)     # (values that all three types hold)
    d = torch.where(d.abs() < 2.0 ** -6, torch.zeros_like(d), d).to(kinds[1]).cuda()
    wide = torch.full((B * (k + 1), pitch), float("nan"), dtype=kinds[0], device="cuda")
    wide[:, :V] = torch.cat([d, d[:, :1]], 1).reshape(-1, V).to(kinds[0])
    ids, u = torch.randint(0, V, (B, k), generator=g, dtype=torch.int32), torch.rand(B, generator=g)
    for alpha in (1.0, 1.5):
        a = torch.full((B, k), alpha)
        n, tok = _run(hs, wide[:, :V], d, ids.cuda(), a.cuda(), u.cuda())
        want_n, want = to.verify(_wide(wide[:, :V]), _wide(d), ids.numpy(), a.numpy(), u.numpy())
        assert (want_n == (k if alpha == 1.0 else 0)).all()
        np.testing.assert_array_equal(n.cpu().numpy(), want_n)
        np.testing.assert_array_equal(tok.cpu().numpy(), want)


def test_the_least_number_of_64_bits(hs):
    """Weights of half of 2^-1074 and more are that number: e^-745 is (2^-1075 is e^-745.13), e^-745.25 is nothing.  At u = 0 the first of them is taken, at alpha 0
    a draft with it stands."""
    depth = torch.tensor([-744.0, -744.5, -744.75, -745.0, -745.25, -745.5, -746.0, -747.0])
    B, V = depth.numel(), 70
    z = torch.full((B, 2, V), -1.0e30)
    z[:, :, 50] = 64.0
    z[:, :, 20] = 64.0 + depth[:, None]
    for token in (20, 50):
        n, tok = _check(hs, z.reshape(2 * B, V), None, torch.full((B, 1), token, dtype=torch.int32), torch.zeros((B, 1)), torch.zeros(B))
        assert n.tolist() == ([1, 1, 1, 1, 0, 0, 0, 0] if token == 20 else [1] * B)
        assert tok[:4, 1].tolist() == [20] * 4 and tok[4:, 1 if token == 50 else 0].tolist() == [50] * 4
