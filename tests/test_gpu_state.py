"""GPU parity of a hybrid target's recurrent layers (hspec_op_chunk_scan) and of the rules of its logits (hspec_op_adjust_logits) against
oracle/state_oracle.py: odd sizes, mixed requests, padded batches, kept rows, values that are not finite, captured calls, other streams."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import state_oracle as so
from oracle import target_oracle as to

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step, relative to the value
# fp16 has the same step for all values below 2^-14, 2^-24: half of it is what they may be off by, whatever their size (bf16 and fp32 go on to 2^-126).
SMALL = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
# What a scan's results may be off by, relative to the sum of the absolute values that enter them.  A product of operands in two bf16 parts: 2^-16 at most and
# some 2^-18 in the mean for each operand's rest and for the product of the remainders; C . B, its weights with x, and C with the state: 9 x 2^-18 where not all
# are off by their most in one direction (these are sums of a hundred terms, or of one whose factors are such sums).  Sums of up to 256 terms in 32 bits:
# 2^8 x 2^-24 = 2^-16.  Convolutions, SiLU, steps and exponentials (arguments up to some 60, so 2^-18 in the power) each a few 2^-20.  Together below 2^-14.
SCAN = 2.0 ** -14


@pytest.fixture(scope="module")
def hs():
    import paper_2609_24197_b200 as m
    m.load_library()
    m.hspec_op_device_status(clear=True)
    return m


def _wide(t):
    return None if t is None else t.double().cpu().numpy()


class Layer:
    """A recurrent layer, its states, and a ragged chunk on the GPU.  Padding rows and places that nobody owns are NaN."""

    def __init__(self, H, P, N, G, new, K=4, dtype=torch.bfloat16, out=None, apart=False, pad=0, seed=0, extra=2, step=-3.0, lead=0):
        g = torch.Generator().manual_seed(991 + seed)
        self.H, self.P, self.N, self.G, self.K, self.new = H, P, N, G, K, list(new)
        self.Di, self.dx, B, T = H * P, H * P + 2 * G * N, len(new), sum(new)
        wide = self.Di + self.dx + (0 if apart else H)
        rows = torch.randn((T + pad, wide), generator=g)
        rows[T:] = float("nan")
        self.T, self.rows_n = T, T + pad
        buf = torch.full((T + pad, wide + lead), float("nan"))
        buf[:, lead:] = rows
        self.rows = buf.to(dtype).cuda()[:, lead:]
        self.dt = None if not apart else torch.randn((T + pad, H), generator=g).cuda()
        u = lambda *s: torch.rand(s, generator=g).cuda()
        self.cw, self.cb = (u(self.dx, K) - 0.5), torch.randn(self.dx, generator=g).cuda() * 0.1
        self.bias, self.A_log, self.D = torch.randn(H, generator=g).cuda() * 0.5 + step, u(H) * 2, torch.randn(H, generator=g).cuda()
        slots = B + extra
        self.slots = torch.randperm(slots, generator=g)[:B].to(torch.int32).cuda()
        self.conv = torch.randn((slots, K - 1, self.dx), generator=g).to(dtype).cuda()
        self.ssm = (torch.randn((slots, H, P, N), generator=g) * 0.5).cuda()
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
        self.y = torch.full((T + pad, self.Di), 7.0, dtype=out or dtype, device="cuda")

    def workspace(self, hs):
        return torch.empty(hs.hspec_chunk_scan_workspace_bytes(self.rows_n, len(self.new), self.Di, self.P, self.N, self.G), dtype=torch.uint8, device="cuda")

    def args(self):
        return (self.rows, self.cw, self.cb, self.bias, self.A_log, self.D, self.cu, self.conv if self.K > 1 else None, self.ssm)

    def run(self, hs, y="own", ws=None, **more):
        more = dict(dt_raw=self.dt, slots=self.slots, **more)
        hs.hspec_op_chunk_scan(*self.args(), self.y if isinstance(y, str) else y, self.workspace(hs) if ws is None else ws, **more)

    def reference(self, sizes=False, **more):
        i = {k: (v.cpu().numpy() if torch.is_tensor(v) else v) for k, v in more.items()}
        i.setdefault("slots", self.slots.cpu().numpy())
        return so.chunk_scan(_wide(self.rows), _wide(self.cw), _wide(self.cb), _wide(self.bias), _wide(self.A_log), _wide(self.D), self.cu.cpu().numpy(),
                             _wide(self.conv), _wide(self.ssm), dt_raw=_wide(self.dt), sizes=sizes, **i)

    def check(self, hs, **more):
        """Runs the layer and compares everything; the references come from the arrays as they were."""
        y, conv, ssm = self.reference(**more)
        sy, _, ss = self.reference(sizes=True, **more)
        before = self.conv.clone(), self.ssm.clone()
        self.run(hs, **more)
        torch.cuda.synchronize()
        got = _wide(self.y)
        assert (got[self.T:] == 7.0).all()
        assert (np.abs(got[:self.T] - y) <= HALF[self.y.dtype] * np.abs(y) + SMALL[self.y.dtype] + SCAN * sy).all()
        np.testing.assert_array_equal(_wide(self.conv), conv)
        assert (np.abs(_wide(self.ssm) - ssm) <= SCAN * ss).all()
        same = (ssm == before[1].double().cpu().numpy()).all(axis=(1, 2, 3))
        assert torch.equal(self.ssm[torch.as_tensor(same)], before[1][torch.as_tensor(same)])            # to the bit
        assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


MIXED = [1, 17, 0, 33, 2, 128, 32, 129, 1, 300]
SHAPES = [(2, 64, 128, 1), (4, 64, 128, 2), (8, 64, 16, 1), (6, 40, 24, 3), (4, 33, 5, 2), (2, 8, 256, 1), (3, 16, 64, 3), (2, 20, 4, 1), (1, 130, 100, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("H,P,N,G", SHAPES)
def test_scan_of_mixed_requests(hs, H, P, N, G, dtype):
    a = Layer(H, P, N, G, MIXED, dtype=dtype, pad=3, seed=P)
    a.check(hs, fresh=torch.tensor([0, 1] * 5, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("K", [1, 2, 3])
@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 1), (6, 40, 24, 3)])
def test_scan_with_a_narrower_convolution(hs, H, P, N, G, K):
    Layer(H, P, N, G, [1, 40, 2, 200, 5], K=K, dtype=torch.float32, seed=K).check(hs)


@pytest.mark.parametrize("new", [[1], [2], [16], [31], [32], [33], [127], [128], [129], [256], [257], [1000], [1] * 40, [9] * 12, [0, 0, 3], [0]])
@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 2), (4, 64, 16, 1)])
def test_scan_lengths(hs, H, P, N, G, new):
    Layer(H, P, N, G, new, dtype=torch.float32, pad=1, seed=len(new), apart=True).check(hs)


@pytest.mark.parametrize("keep", [0, 1, 2, 3, 7, 31, 32, 33, 100, 128, 130, 255, 256, 999])
@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 1), (2, 40, 24, 1)])
def test_scan_keeps_as_many_rows_as_it_is_told(hs, H, P, N, G, keep):
    for with_y in (True, False):
        a = Layer(H, P, N, G, [300, 32, 140, 1, 5], dtype=torch.float32, seed=keep)
        n = torch.tensor([keep, keep, keep - 1, keep, 0], dtype=torch.int32, device="cuda")
        more = dict(keep=n, keep_more=0, fresh=torch.tensor([0, 1, 0, 0, 1], dtype=torch.int32, device="cuda"))
        if with_y:
            a.check(hs, **more)
            continue
        _, conv, ssm = a.reference(**more)
        size = a.reference(sizes=True, **more)[2]
        a.run(hs, y=None, **more)
        np.testing.assert_array_equal(_wide(a.conv), conv)
        assert (np.abs(_wide(a.ssm) - ssm) <= SCAN * size).all()


def test_scan_counts_of_drafts_with_the_token_in_front(hs):
    a = Layer(2, 64, 128, 1, [9, 9, 9, 9], seed=3)
    n = torch.tensor([0, 3, 8, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    a.check(hs, keep=n, keep_more=1)


@pytest.mark.parametrize("H,P,N,G", [(4, 64, 128, 1), (4, 64, 16, 1)])
def test_scan_of_a_verification_and_its_commit(hs, H, P, N, G):
    """Looking at a block and then committing the accepted rows leaves the states that these rows alone leave, and no other call's."""
    a = Layer(H, P, N, G, [17] * 5, seed=8)
    conv, ssm = a.conv.clone(), a.ssm.clone()
    a.check(hs, keep=torch.zeros(5, dtype=torch.int32, device="cuda"))
    assert torch.equal(a.conv, conv) and torch.equal(a.ssm, ssm)
    accepted = torch.tensor([0, 16, 3, 9, 1], dtype=torch.int32, device="cuda")
    a.run(hs, y=None, keep=accepted, keep_more=1)
    whole = Layer(H, P, N, G, [17] * 5, seed=8)
    _, conv, ssm = whole.reference(keep=accepted, keep_more=1)
    np.testing.assert_array_equal(_wide(a.conv), conv)
    assert (np.abs(_wide(a.ssm) - ssm) <= SCAN * whole.reference(sizes=True, keep=accepted, keep_more=1)[2]).all()


@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 1), (6, 40, 24, 3)])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16), (torch.float16, torch.float16)])
def test_scan_of_rows_at_odd_addresses(hs, H, P, N, G, dtype, out):
    """Rows at odd addresses and pitches, y with an odd pitch of its own."""
    a = Layer(H, P, N, G, [3, 200, 20], dtype=dtype, out=out, seed=5, lead=3)
    buf = torch.full((a.rows_n, a.Di + 5), 7.0, dtype=out, device="cuda")
    a.y = buf[:, 3:3 + a.Di]
    a.check(hs)
    assert (buf[:, :3] == 7.0).all() and (buf[:, 3 + a.Di:] == 7.0).all()


@pytest.mark.parametrize("step", [-30.0, 4.0])
def test_scan_of_tiny_and_of_long_steps(hs, step):
    """Steps near zero (nothing decays, nothing is added) and of several units (all decays within a row or two)."""
    Layer(2, 64, 128, 1, [2, 20, 260], dtype=torch.float32, step=step, seed=2).check(hs)
    Layer(2, 40, 24, 1, [2, 20, 260], dtype=torch.float32, step=step, seed=2).check(hs)


@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 1), (2, 40, 24, 1)])
@pytest.mark.parametrize("new,where", [([20], 5), ([20], 18), ([300], 40), ([300], 130), ([300], 299), ([300, 30], 3), ([5, 30], 2)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_scan_of_a_value_that_is_not_finite_reaches_no_row_in_front_of_it(hs, H, P, N, G, new, where, value):
    a, b = (Layer(H, P, N, G, new, dtype=torch.float32, seed=1) for _ in range(2))
    a.rows[where, a.Di + 3] = value                            # a channel of x: the first head's
    a.run(hs)
    torch.cuda.synchronize()
    got = a.y.double().cpu()
    want, size = b.reference()[0], b.reference(sizes=True)[0]
    ok = torch.isfinite(got)
    assert ok[:where].all() and not ok[where, 3]
    touched = torch.zeros(a.Di, dtype=torch.bool)
    touched[3] = True
    assert ok[:, ~touched].all()                               # no other channel, and no other request
    # (rows in front may be summed in another order than they were without it: the same distance from the formula, not the same bits)
    sure = ok.numpy()
    assert (np.abs(got.numpy() - want) <= HALF[torch.float32] * np.abs(want) + SCAN * size)[sure].all()
    assert not ok[where:new[0], 3].any() if where < new[0] else True
    s = torch.isfinite(a.ssm).all(dim=3).cpu()
    bad = ~s
    assert bad.sum() == 1 and bad[int(a.slots[0])][0, 3]


@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 1), (2, 40, 24, 1), (2, 64, 16, 2)])
@pytest.mark.parametrize("new,where", [([20], 5), ([20], 18), ([32], 16), ([300], 40), ([300], 128), ([300], 299), ([300, 30], 3), ([5, 30], 2), ([2, 1], 1)])
@pytest.mark.parametrize("place", ["z", "x", "B", "C", "dt"])
def test_scan_of_nan_in_a_row_that_is_not_kept(hs, H, P, N, G, new, where, place):
    a, b = (Layer(H, P, N, G, new, dtype=torch.float32, seed=13) for _ in range(2))
    keep = torch.tensor([where] + new[1:], dtype=torch.int32, device="cuda")
    a.rows[where, {"z": 1, "x": a.Di + 1, "B": 2 * a.Di + 1, "C": 2 * a.Di + G * N + 1, "dt": -1}[place]] = float("nan")
    y, conv, ssm = b.reference(keep=keep)
    sy, _, ss = b.reference(sizes=True, keep=keep)
    for with_y in ("own", None):
        a.conv.copy_(b.conv), a.ssm.copy_(b.ssm)
        a.run(hs, y=with_y, keep=keep)
        torch.cuda.synchronize()
        assert (np.abs(_wide(a.ssm) - ssm) <= SCAN * ss).all()
        np.testing.assert_array_equal(_wide(a.conv), conv)
    got, mine = _wide(a.y), np.r_[0:where, new[0]:sum(new)]
    assert (np.abs(got - y) <= HALF[torch.float32] * np.abs(y) + SCAN * sy)[mine].all()
    assert not np.isfinite(got[where]).all()


def test_scan_of_nan_in_places_that_are_not_its_own(hs):
    """Slots that no request has, states of fresh requests, rows behind the last one."""
    for shape in ((2, 64, 128, 1), (2, 40, 24, 1)):
        a = Layer(*shape, [40, 5, 200], dtype=torch.float32, pad=6, seed=4)
        own = a.slots.long()
        a.ssm[own[1]], a.conv[own[1]] = float("nan"), float("nan")
        others = [i for i in range(a.ssm.shape[0]) if i not in own.tolist()]
        a.ssm[others], a.conv[others] = float("nan"), float("nan")
        fresh = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
        a.run(hs, fresh=fresh)
        assert torch.isfinite(a.y[:a.T]).all() and (a.y[a.T:] == 7.0).all()
        assert torch.isfinite(a.ssm[own]).all() and torch.isnan(a.ssm[others]).all()


@pytest.mark.parametrize("H,P,N,G", [(2, 64, 128, 1), (2, 40, 24, 1)])
def test_scan_counts_bad_slots_and_offsets(hs, H, P, N, G):
    a = Layer(H, P, N, G, [3, 40, 3, 0], dtype=torch.float32, seed=6)
    conv, ssm = a.conv.clone(), a.ssm.clone()
    slots = torch.tensor([-1, a.ssm.shape[0], 0, -7], dtype=torch.int32, device="cuda")
    want = a.reference(slots=slots)
    hs.hspec_op_chunk_scan(*a.args(), a.y, a.workspace(hs), slots=slots)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 2                      # (a request without rows needs no slot)
    np.testing.assert_array_equal(_wide(a.conv), want[1])
    assert torch.equal(a.ssm[1:], ssm[1:]) and torch.equal(a.conv[1:], conv[1:]) and torch.isfinite(a.y).all()
    a.cu.copy_(torch.tensor([0, 3, -5, 2 ** 31 - 1, 46], dtype=torch.int32))
    a.run(hs)
    torch.cuda.synchronize()
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] >= 2


def test_scan_of_thousands_of_requests(hs):
    a = Layer(2, 64, 128, 1, [1] * 3000, dtype=torch.float32, pad=7, seed=9)
    a.check(hs)
    Layer(2, 8, 16, 1, [2, 0, 1] * 900, dtype=torch.float32, seed=9).check(hs)


def test_scan_without_any_row(hs):
    for shape in ((2, 64, 128, 1), (2, 40, 24, 1)):
        a = Layer(*shape, [0, 0], seed=14)
        conv, ssm = a.conv.clone(), a.ssm.clone()
        a.run(hs, fresh=torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
        own = int(a.slots[1])
        conv[own], ssm[own] = 0, 0
        assert torch.equal(a.conv, conv) and torch.equal(a.ssm, ssm)


@pytest.mark.parametrize("H,P,N,G,new", [(2, 64, 128, 1, [40000, 20, 29990, 1]), (2, 64, 128, 1, [2] * 34998 + [1, 1]), (8, 64, 16, 1, [3] * 20000 + [9000, 2, 1010])])
def test_scan_behind_2_to_the_31_elements(hs, H, P, N, G, new):
    """Rows, outputs and states whose places pass 32 bits: the bits that they have in small arrays."""
    B, T = len(new), sum(new)
    a = Layer(H, P, N, G, new[-4:], seed=15)                   # (the weights)
    width = a.rows.shape[1]
    g = torch.Generator(device="cuda").manual_seed(15)
    pitch = 2 ** 31 // T // 16 * 16 + 32
    far, far_y = (torch.empty((T, pitch), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    near, near_y = torch.empty((T, (width + 15) // 16 * 16), dtype=torch.bfloat16, device="cuda"), torch.empty((T, H * P), dtype=torch.bfloat16, device="cuda")
    near.normal_(generator=g)
    far[:, :width] = near[:, :width]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    conv = torch.randn((B, a.K - 1, a.dx), dtype=torch.float32, device="cuda", generator=g).to(torch.bfloat16)
    ws = torch.empty(hs.hspec_chunk_scan_workspace_bytes(T, B, a.Di, P, N, G), dtype=torch.uint8, device="cuda")
    fresh = torch.ones(B, dtype=torch.int32, device="cuda")
    fresh[-3:] = 0
    last = torch.randn((3, H, P, N), device="cuda", generator=g)
    results = []
    n_far = 2 ** 31 // (H * P * N) + B
    for rows, y, n in ((near, near_y, B), (far, far_y, n_far)):
        ssm = torch.empty((n, H, P, N), device="cuda")
        ssm[n - 3:] = last
        slots = torch.arange(n - B, n, dtype=torch.int32, device="cuda")
        carried = conv.clone() if n == B else torch.cat([torch.zeros((n - B, a.K - 1, a.dx), dtype=conv.dtype, device="cuda"), conv])
        hs.hspec_op_chunk_scan(rows[:, :width], a.cw, a.cb, a.bias, a.A_log, a.D, cu, carried, ssm, y[:, :a.Di], ws, slots=slots, fresh=fresh)
        results.append((y[:, :a.Di].clone(), carried[n - B:].clone(), ssm[n - B:].clone()))
        del ssm
    for x, y in zip(*results):
        assert torch.equal(x, y) and torch.isfinite(x).all()
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


def test_scan_of_a_prompt_in_pieces(hs):
    """A prompt at once, in pieces and token by token: the same outputs and states within what both may be off by."""
    whole = Layer(2, 64, 128, 1, [290], dtype=torch.float32, seed=11)
    y, _, ssm = whole.reference()
    sy, _, ss = whole.reference(sizes=True)
    for cuts in ((0, 290), (0, 1, 2, 290), (0, 128, 160, 161, 290), tuple(range(0, 291, 29)), (0, 200, *range(201, 291))):
        a = Layer(2, 64, 128, 1, [290], dtype=torch.float32, seed=11)
        ws = a.workspace(hs)
        for lo, hi in zip(cuts, cuts[1:]):
            cu = torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda")
            hs.hspec_op_chunk_scan(a.rows[lo:hi], a.cw, a.cb, a.bias, a.A_log, a.D, cu, a.conv, a.ssm, a.y[lo:hi], ws, slots=a.slots)
        torch.cuda.synchronize()
        # (as many states are stored and taken up again as there are pieces: a rounding each is far inside)
        assert (np.abs(_wide(a.y) - y) <= HALF[torch.float32] * np.abs(y) + SCAN * sy).all()
        assert (np.abs(_wide(a.ssm) - ssm) <= SCAN * ss).all()


def test_scan_captured_follows_its_arrays(hs):
    a = Layer(2, 64, 128, 1, [60, 60, 60], pad=20, seed=12)
    b = Layer(2, 64, 128, 1, [60, 60, 60], pad=20, seed=12)
    ws, keep, fresh = a.workspace(hs), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hspec_op_chunk_scan(*a.args(), a.y, ws, slots=a.slots, keep=keep, keep_more=1, fresh=fresh)
    for new, kept, first in (([60, 60, 60], [59, 3, 0], [0, 0, 1]), ([1, 0, 170], [0, 0, 129], [0, 1, 0]), ([5, 100, 33], [9, 40, -1], [0, 0, 0])):
        for x in (a, b):
            x.cu.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
            x.y.fill_(7.0)
        b.rows.nan_to_num_(0.0), a.rows.nan_to_num_(0.0)
        keep.copy_(torch.tensor(kept, dtype=torch.int32)), fresh.copy_(torch.tensor(first, dtype=torch.int32))
        graph.replay()
        b.run(hs, keep=keep, keep_more=1, fresh=fresh)
        torch.cuda.synchronize()
        assert torch.equal(a.y, b.y) and torch.equal(a.ssm, b.ssm) and torch.equal(a.conv, b.conv)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


def test_scan_on_two_streams(hs):
    layers = [Layer(2, 64, 128, 1, [200, 20, 1], dtype=torch.float32, seed=s) for s in (20, 21)]
    again = [Layer(2, 64, 128, 1, [200, 20, 1], dtype=torch.float32, seed=s) for s in (20, 21)]
    streams = [torch.cuda.Stream() for _ in layers]
    spaces = [x.workspace(hs) for x in layers]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, s, w in zip(layers, streams, spaces):
            with torch.cuda.stream(s):
                x.run(hs, ws=w)
    torch.cuda.synchronize()
    for x, y in zip(layers, again):
        for _ in range(3):
            y.run(hs)
        torch.cuda.synchronize()
        assert torch.equal(x.y, y.y) and torch.equal(x.ssm, y.ssm) and torch.equal(x.conv, y.conv)


# ---------------------------------------------------------------------------------------------------- the rules of logits

def _rules(V, rows, seed=0, dtype=torch.float32, history=50, wide=60, drafts=6, biases=5, masks=3, pad=0, lead=0):
    g = torch.Generator().manual_seed(77 + seed)
    B, T = len(rows), sum(rows)
    buf = torch.randn((T + pad, V + lead), generator=g) * 3
    z = buf.to(dtype).cuda()[:, lead:]
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, dtype=torch.int32).cuda()
    some = max(1, min(V, 12))                                  # (few tokens, so that they come back)
    return z, dict(cu_q=torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32).cuda(), history=ints(0, some, B, wide),
                   history_lens=ints(0, history + 1, B), prompt_lens=ints(0, 4, B), drafts=ints(0, some, B, drafts),
                   repetition=torch.rand(B, generator=g).cuda() + 0.6, frequency=torch.randn(B, generator=g).cuda() * 0.3,
                   presence=torch.randn(B, generator=g).cuda(), bias_ids=ints(0, V, B, biases), bias_values=torch.randn((B, biases), generator=g).cuda(),
                   bias_counts=ints(0, biases + 1, B), mask=ints(-2 ** 31, 2 ** 31 - 1, masks, (V + 31) // 32 + 1), mask_rows=ints(-1, masks, T + pad))


def _check_rules(hs, z, rules, out=None, same=False):
    rules = {k: v for k, v in rules.items() if v is not None}
    host = {k: v.cpu().numpy() for k, v in rules.items()}
    want = so.adjust_logits(_wide(z), **host)
    used = z.shape[0] if "cu_q" not in rules else int(rules["cu_q"][-1])
    out = z if same else torch.full(z.shape, 7.0, dtype=out or z.dtype, device="cuda")
    hs.hspec_op_adjust_logits(z, out, **rules)
    torch.cuda.synchronize()
    got = _wide(out)
    if not same:
        assert (got[used:] == 7.0).all()
    got, want = got[:used], want[:used]
    np.testing.assert_array_equal(np.isneginf(got), np.isneginf(want))
    on = np.isfinite(want)
    # seven operations in 32 bits, each off by 2^-24 of the largest value on the way: |z| r, f count + p, the biases
    count = (host["history"].shape[1] if "history" in host else 0) + (host["drafts"].shape[1] if "drafts" in host else 0)
    top = lambda k: np.abs(host[k]).max() if k in host else 0.0
    size = np.abs(_wide(z)[:used][on] if not same else want[on]) * 2.0 + np.abs(want[on]) + top("frequency") * count + top("presence") + 8 * top("bias_values")
    assert (np.abs(got[on] - want[on]) <= HALF[out.dtype] * np.abs(want[on]) + SMALL[out.dtype] + 8 * 2.0 ** -24 * size).all()
    return out


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float16, torch.float16),
                                       (torch.float16, torch.float32)])
@pytest.mark.parametrize("V,rows,lead", [(1, [1, 2], 0), (7, [3, 0, 1], 0), (31, [2], 1), (1000, [1, 9, 33, 0, 4], 0), (4097, [40, 3], 3), (8191, [2, 2], 0), (50021, [7, 1], 0)])
def test_rules_together(hs, V, rows, lead, dtype, out):
    z, rules = _rules(V, rows, dtype=dtype, pad=2, lead=lead, seed=V)
    _check_rules(hs, z, rules, out)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


@pytest.mark.parametrize("left_out", ["history", "history_lens", "prompt_lens", "drafts", "repetition", "frequency", "presence", "bias_ids", "bias_counts", "mask", "cu_q",
                                      "penalties", "all but mask", "all but bias", "all"])
def test_rules_one_by_one(hs, left_out):
    z, rules = _rules(3001, [1] * 6 if left_out == "cu_q" else [4, 2, 9], seed=3)
    gone = {"bias_ids": ["bias_ids", "bias_values", "bias_counts"], "mask": ["mask", "mask_rows"], "penalties": ["repetition", "frequency", "presence"],
            "all but mask": [k for k in rules if k not in ("cu_q", "mask", "mask_rows")], "all but bias": [k for k in rules if k != "cu_q" and "bias" not in k],
            "all": [k for k in rules if k != "cu_q"]}.get(left_out, [left_out])
    for place in (False, True):
        zz, more = z.clone(), {k: (None if k in gone else v) for k, v in rules.items()}
        if place:
            apart = torch.empty_like(zz)
            hs.hspec_op_adjust_logits(z, apart, **{k: v for k, v in more.items() if v is not None})
            hs.hspec_op_adjust_logits(zz, zz, **{k: v for k, v in more.items() if v is not None})
            assert torch.equal(zz, apart)
        else:
            _check_rules(hs, zz, more)


def test_rules_mask_without_rows_of_its_own(hs):
    z, rules = _rules(500, [3, 2], seed=4, masks=5)
    rules["mask_rows"] = None
    _check_rules(hs, z, rules)


@pytest.mark.parametrize("place", [False, True])
def test_rules_of_values_that_are_not_finite(hs, place):
    """What is forbidden is -infinity whatever it was; a row may be left without anything; infinities and NaN that are allowed go their way."""
    z = torch.tensor([[float("nan"), float("inf"), -float("inf"), 1.0, 2.0, -1e30, 3e38, 0.0]] * 3, device="cuda")
    mask = torch.tensor([[0], [0b11111000], [0xff]], dtype=torch.int64).to(torch.int32).cuda()
    out = z.clone() if place else torch.empty_like(z)
    hs.hspec_op_adjust_logits(out if place else z, out, mask=mask)
    assert torch.isneginf(out[0]).all() and torch.isneginf(out[1, :3]).all()
    assert torch.equal(out[1, 3:], z[1, 3:]) and torch.equal(out[2].nan_to_num(5.0), z[2].nan_to_num(5.0))


def test_rules_many_tokens_of_one_kind_and_long_texts(hs):
    V = 20011
    z, rules = _rules(V, [3, 1], seed=5, wide=70000, history=70000, biases=1024)
    rules["history"].copy_(torch.randint(0, V, rules["history"].shape, generator=torch.Generator().manual_seed(1), dtype=torch.int32))
    rules["history"][0, :60000] = 77
    rules["history_lens"].copy_(torch.tensor([70000, 65537], dtype=torch.int32))
    rules["bias_ids"][:] = torch.arange(1024, device="cuda", dtype=torch.int32) % 7          # the same few tokens again and again
    rules["bias_counts"] = None
    rules["frequency"].mul_(1e-3)
    z1 = z.clone()
    want = so.adjust_logits(_wide(z), **{k: v.cpu().numpy() for k, v in rules.items() if v is not None})
    hs.hspec_op_adjust_logits(z, z1, **{k: v for k, v in rules.items() if v is not None})
    on = np.isfinite(want)
    # (a token's 147 biases are added one by one: 147 roundings of their sum of at most 147 x 5)
    assert (np.isneginf(_wide(z1)) == ~on).all() and (np.abs(_wide(z1)[on] - want[on]) <= 2.0 ** -24 * (8 * (np.abs(want[on]) + 100) + 147 * 735)).all()


def test_rules_count_what_cannot_be(hs):
    z, rules = _rules(100, [2, 2], seed=6)
    for k in ("bias_ids", "bias_values", "bias_counts", "mask", "mask_rows"):
        rules[k] = None
    rules["history"][0, :3] = torch.tensor([-1, 100, 2 ** 31 - 1], dtype=torch.int32)
    rules["history_lens"].copy_(torch.tensor([10, 61], dtype=torch.int32))
    rules["prompt_lens"].zero_()
    rules["drafts"][1, 0] = -5
    _check_rules(hs, z, rules)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 5
    z, rules = _rules(100, [2, 2], seed=6)
    rules["mask_rows"].copy_(torch.tensor([-2, 3, 0, -1], dtype=torch.int32))
    rules["bias_ids"][0, :2], rules["bias_counts"] = torch.tensor([-1, 100], dtype=torch.int32), None
    _check_rules(hs, z, rules)
    assert hs.hspec_op_device_status(clear=True)["bad_inputs"] == 4


def test_rules_clamp_what_leaves_fp16(hs):
    z = torch.tensor([[60000.0, -60000.0, 1.0]], dtype=torch.float16, device="cuda")
    r = torch.tensor([2.0], device="cuda")
    out = torch.empty_like(z)
    hs.hspec_op_adjust_logits(z, out, history=torch.tensor([[1]], dtype=torch.int32, device="cuda"), repetition=r, bias_ids=torch.tensor([[0]], dtype=torch.int32, device="cuda"),
                              bias_values=torch.tensor([[1e5]], device="cuda"))
    assert out.tolist() == [[65504.0, -65504.0, 1.0]]
    assert hs.hspec_op_device_status(clear=True)["f16_range_events"] == 2


def test_rules_behind_2_to_the_31_elements(hs):
    z, rules = _rules(1000, [200, 300, 20], seed=10, dtype=torch.bfloat16, drafts=30)
    out = torch.empty_like(z)
    hs.hspec_op_adjust_logits(z, out, **rules)
    far, far_out = (torch.empty((520, 2 ** 31 // 520 // 8 * 8 + 16), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far[:, :1000] = z
    hs.hspec_op_adjust_logits(far[:, :1000], far_out[:, :1000], **rules)
    assert torch.equal(far_out[:, :1000], out)
    hs.hspec_op_adjust_logits(far[:, :1000], far[:, :1000], **rules)
    assert torch.equal(far[:, :1000], out)


def test_rules_captured_and_on_another_stream(hs):
    z, rules = _rules(9001, [5, 1, 17], seed=7, dtype=torch.bfloat16, drafts=20)
    out = torch.empty_like(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hs.hspec_op_adjust_logits(z, out, **rules)
    for seed in (8, 9):
        z2, r2 = _rules(9001, [5, 1, 17] if seed == 8 else [0, 20, 3], seed=seed, dtype=torch.bfloat16, drafts=20)
        z.copy_(z2)
        for k, v in r2.items():
            rules[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        other = torch.empty_like(z)
        with torch.cuda.stream(s):
            hs.hspec_op_adjust_logits(z, other, **rules)
        s.synchronize()
        assert torch.equal(out, other)
        _check_rules(hs, z, rules)


# ---------------------------------------------------------------------------------------------------- as they are used

def test_iterations_of_a_hybrid_target(hs):
    """Scan, LM head, rules, verification and the commit of what stands, all of it one captured graph over several iterations: after each the states are
    those that the accepted tokens leave, one after another, in 64 bits."""
    B, K, V, H, P, N, G = 3, 6, 301, 2, 64, 128, 1
    g = torch.Generator().manual_seed(31)
    Di = H * P
    table = torch.randn((V, 2 * Di + 2 * G * N + H), generator=g).to(torch.bfloat16).cuda()                # a token's rows
    a = Layer(H, P, N, G, [K + 1] * B, seed=30)
    head = (torch.randn((V, Di), generator=g) * 0.1).to(torch.bfloat16).cuda()
    rows_ids, ids = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((B * (K + 1),), (B, K)))
    logits, ruled = (torch.zeros((B * (K + 1), V), device="cuda") for _ in range(2))
    draft_logits = torch.zeros((B, K, V), device="cuda")
    alpha, u = torch.zeros((B, K), device="cuda"), torch.zeros(B, device="cuda")
    n, tokens, none = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, K + 1), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    history, lens = torch.zeros((B, 200), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    rules = dict(repetition=torch.tensor([1.2, 1.0, 1.1], device="cuda"), frequency=torch.tensor([0.1, 0.0, 0.2], device="cuda"))
    mask, rule = torch.randint(-2 ** 31, 2 ** 31 - 1, (4, 10), generator=g, dtype=torch.int32).cuda(), torch.zeros(B * (K + 1), dtype=torch.int32, device="cuda")
    rule.copy_(torch.randint(-1, 4, rule.shape, generator=g))
    ws, vws = a.workspace(hs), torch.empty(hs.hspec_verify_workspace_bytes(B, K), dtype=torch.uint8, device="cuda")

    def scan(y, **more):
        hs.hspec_op_chunk_scan(table[rows_ids.long()], a.cw, a.cb, a.bias, a.A_log, a.D, a.cu, a.conv, a.ssm, y, ws, slots=a.slots, **more)

    def iteration():
        scan(a.y, keep=none)
        hs.hspec_op_gemm(a.y, head, logits, splits=1)
        hs.hspec_op_adjust_logits(logits, ruled, cu_q=a.cu, history=history, history_lens=lens, drafts=ids, mask=mask, mask_rows=rule, **rules)
        hs.hspec_op_verify(ruled, draft_logits, ids, alpha, u, n, tokens, vws, cu_q=a.cu)
        scan(None, keep=n, keep_more=1)

    iteration()                                                # (the first call of an operator sets its kernels up)
    fresh = Layer(H, P, N, G, [K + 1] * B, seed=30)
    a.ssm.copy_(fresh.ssm), a.conv.copy_(fresh.conv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iteration()
    layer = [_wide(x) for x in (a.cw, a.cb, a.bias, a.A_log, a.D)]
    conv, ssm = _wide(a.conv), _wide(a.ssm)
    size = np.abs(ssm)
    seq, counts = [[5], [6], [7]], []
    for it in range(6):
        z = torch.randn((B, K, V), generator=g)
        d = torch.stack([torch.multinomial(torch.softmax(z[b], 1), 1, generator=g).squeeze(1) for b in range(B)])
        draft_logits.copy_(z), ids.copy_(d.to(torch.int32)), alpha.copy_(torch.rand((B, K), generator=g) * 0.5), u.copy_(torch.rand(B, generator=g))
        rows_ids.copy_(torch.cat([torch.tensor([seq[b][-1]] + d[b].tolist()) for b in range(B)]).to(torch.int32))
        for b in range(B):
            history[b, :len(seq[b])] = torch.tensor(seq[b], dtype=torch.int32)
        lens.copy_(torch.tensor([len(s) for s in seq], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = so.adjust_logits(_wide(logits), a.cu.cpu().numpy(), history.cpu().numpy(), lens.cpu().numpy(), None, ids.cpu().numpy(), _wide(rules["repetition"]),
                                _wide(rules["frequency"]), mask=mask.cpu().numpy(), mask_rows=rule.cpu().numpy())
        np.testing.assert_array_equal(np.isneginf(want), np.isneginf(_wide(ruled)))
        on = np.isfinite(want)
        np.testing.assert_allclose(_wide(ruled)[on], want[on], rtol=2.0 ** -20, atol=2.0 ** -18)
        want_n, want_t = to.verify(_wide(ruled), _wide(draft_logits), *(x.cpu().numpy() for x in (ids, alpha, u, a.cu)))
        np.testing.assert_array_equal(n.cpu().numpy(), want_n)
        np.testing.assert_array_equal(tokens.cpu().numpy(), want_t)
        for b in range(B):
            stands = int(n[b]) + 1
            part = table[rows_ids.long()][b * (K + 1):b * (K + 1) + stands].double().cpu().numpy()
            kw = dict(slots=[int(a.slots[b])])
            _, c2, s2 = so.chunk_scan(part, *layer, [0, stands], conv, ssm, **kw)
            size = so.chunk_scan(part, *layer, [0, stands], conv, size, sizes=True, **kw)[2]
            conv, ssm = c2, s2
            got = [t for t in tokens[b].tolist() if t >= 0]
            seq[b] += got
            counts.append(len(got))
        np.testing.assert_array_equal(_wide(a.conv), conv)
        assert (np.abs(_wide(a.ssm) - ssm) <= SCAN * size).all()
    assert max(counts) > 1 and hs.hspec_op_device_status(clear=True)["bad_inputs"] == 0


FIRST_CALL = """
import sys, torch
import paper_2609_24197_b200 as hs
sys.path.insert(0, "tests")
import test_gpu_state as t
a, b = (t.Layer(2, 64, 128, 1, [3, 200, 20], dtype=torch.float32, seed=40) for _ in range(2))
z, rules = t._rules(5001, [3, 0, 9], seed=41)
out, ws = torch.empty_like(z), a.workspace(hs)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    if sys.argv[1] == "scan": a.run(hs, ws=ws)
    else: hs.hspec_op_adjust_logits(z, out, **rules)
graph.replay()
torch.cuda.synchronize()
if sys.argv[1] == "scan":
    b.run(hs)
    torch.cuda.synchronize()
    assert torch.equal(a.y, b.y) and torch.equal(a.ssm, b.ssm)
else:
    t._check_rules(hs, z, rules)
"""


@pytest.mark.parametrize("what", ["scan", "rules"])
def test_the_first_call_of_a_process_may_be_a_captured_one(what):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALL, what], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-1500:]
