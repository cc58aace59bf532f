"""Edges of hspec_op_chunk_scan on the GPU: rows that are no numbers, narrow states, long chains of rows, narrow convolutions, errors that others left."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from test_gpu_state import HALF, SCAN, Layer, _wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hs():
    import paper_2609_24197_b200 as m
    m.load_library()
    m.hspec_op_device_status(clear=True)
    return m


def _near(got, want, size, half=0.0, bound=SCAN):
    return np.abs(got - want) <= half * np.abs(want) + bound * size


# chunks of 128 rows, blocks of up to 32, row after row
WAYS = [((2, 64, 128, 1), [300], 40), ((2, 64, 128, 1), [300], 130), ((2, 64, 128, 1), [300], 299), ((2, 64, 128, 1), [20], 5), ((2, 64, 128, 1), [20], 18),
        ((2, 40, 24, 1), [300], 130), ((4, 64, 16, 1), [300], 40)]


# outputs of 16 and of 32 bits take their operands in different numbers of parts
OUT = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("shape,new,where", WAYS)
def test_a_row_without_numbers_reaches_no_row_in_front_of_it(hs, shape, new, where, out):
    """All of a row NaN: gate, x, B, C and dt.  Every row is kept."""
    a, b = (Layer(*shape, new, dtype=torch.float32, out=out, seed=50) for _ in range(2))
    a.rows[where] = float("nan")
    a.run(hs)
    torch.cuda.synchronize()
    got, want, size = _wide(a.y), b.reference()[0], b.reference(sizes=True)[0]
    assert _near(got, want, size, HALF[out])[:where].all()
    assert not np.isfinite(got[where:]).any()
    assert not torch.isfinite(a.ssm[a.slots.long()]).any()


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("shape,new,where", WAYS)
@pytest.mark.parametrize("behind", [1, 20, -2])
@pytest.mark.parametrize("value,step", [(float("inf"), float("nan")), (float("nan"), float("inf"))])
def test_x_and_a_step_that_are_no_numbers_in_different_rows(hs, shape, new, where, behind, value, step, out):
    a, b = (Layer(*shape, new, dtype=torch.float32, out=out, seed=51) for _ in range(2))
    H, P, N, G = shape
    at = min(where + behind, new[0] - 1)
    a.rows[where, a.Di + 3] = value                            # a channel of x of the first head
    a.rows[at, 2 * a.Di + 2 * G * N] = step                    # that head's step
    a.run(hs)
    torch.cuda.synchronize()
    got, want, size = _wide(a.y), b.reference()[0], b.reference(sizes=True)[0]
    near = _near(got, want, size, HALF[out])
    assert near[:min(where, at)].all() and near[:, P:].all()   # rows in front of both, and all other heads
    others = [p for p in range(P) if p != 3]
    assert near[:at, others].all()                             # the head's other channels, up to its step
    assert not np.isfinite(got[where:, 3]).any() and not np.isfinite(got[at + 1:, :P]).any()


@pytest.mark.parametrize("H,P,N,G", [(2, 65, 4, 1), (1, 128, 3, 1), (2, 65, 1, 2), (4, 128, 4, 2), (1, 256, 3, 1), (1, 200, 1, 1), (2, 64, 2, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_states_of_up_to_four_elements_and_wide_heads(hs, H, P, N, G, dtype):
    new = [1, 17, 0, 33, 70]
    keep = torch.tensor([1, 9, 0, 33, 64], dtype=torch.int32, device="cuda")
    Layer(H, P, N, G, new, dtype=dtype, pad=3, seed=52).check(hs)
    a = Layer(H, P, N, G, new, dtype=dtype, seed=53)
    _, conv, ssm = a.reference(keep=keep)
    size = a.reference(sizes=True, keep=keep)[2]
    a.run(hs, y=None, keep=keep)
    np.testing.assert_array_equal(_wide(a.conv), conv)
    assert _near(_wide(a.ssm), ssm, size).all()


LEFT_ERROR = """
import sys, ctypes, torch
import paper_2609_24197_b200 as hs
sys.path.insert(0, "tests")
import test_gpu_state as t
a, b = (t.Layer(2, 64, 128, 1, [300, 20], dtype=torch.float32, seed=54) for _ in range(2))
for x in (b, a):
    ws = x.workspace(hs)
    if x is a:                                                 # a call on the legacy stream fails while a stream that waits for that one is captured
        cudart = ctypes.CDLL("libcudart.so.12")
        side, none = ctypes.c_void_p(), ctypes.c_void_p()
        assert cudart.cudaStreamCreate(ctypes.byref(side)) == 0 and cudart.cudaStreamBeginCapture(side, 0) == 0
        assert hs.hspec_op_device_status()["rc"] == -6
        cudart.cudaStreamEndCapture(side, ctypes.byref(none))
        cudart.cudaGetLastError()
    x.run(hs, ws=ws)
torch.cuda.synchronize()
assert torch.equal(a.y, b.y) and torch.equal(a.ssm, b.ssm) and torch.equal(a.conv, b.conv)
"""


def test_an_error_that_another_call_left_does_not_end_the_scan_in_the_middle():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", LEFT_ERROR], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-1500:]


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("shape,new,where", [((2, 64, 128, 1), [300], 130), ((2, 64, 128, 1), [300, 9], 250), ((2, 64, 128, 1), [20], 5), ((2, 40, 24, 1), [40], 9)])
@pytest.mark.parametrize("place", ["x", "C"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_value_that_is_no_number_reaches_as_far_as_the_convolution(hs, shape, new, where, place, value, K, out):
    a, b = (Layer(*shape, new, K=K, dtype=torch.float32, out=out, seed=55) for _ in range(2))
    H, P, N, G = shape
    a.rows[where, a.Di + (3 if place == "x" else a.Di + G * N + 5)] = value
    a.run(hs)
    torch.cuda.synchronize()
    got, want, size = _wide(a.y), b.reference()[0], b.reference(sizes=True)[0]
    near = _near(got, want, size, HALF[out])
    assert near[:where].all() and near[new[0]:].all()
    if place == "C":                                           # nothing of it stays in the state
        assert near[where + K:].all() and not np.isfinite(got[where]).any()
        assert _near(_wide(a.ssm), b.reference()[2], b.reference(sizes=True)[2]).all()
    else:                                                      # from its row on, in its channel
        assert np.delete(near, 3, axis=1).all() and not np.isfinite(got[where:new[0], 3]).any()


# Row after row, relative to the sum of the absolute values that enter a result, in roundings of 32 bits: a convolved value 5 for its terms and 7 for SiLU (two
# units for its exponential and one for the argument's product at |v| of a few, its sum, its division); a step 4; a decay as much as its step and its rate,
# 9 times c e^c <= 0.37, however many rows there are; the state 8 (one for each of up to eight rows; two where there are more, which carry the rest on).
# A state has x, B and the step: 40 of them.  An output has C beside these, a sum of 16 products in a lane, one of up to 16 lanes, Dskip, and its gate with
# 8: 40 + 12 + 20 + 2 + 8, below 84.
STATE_ROWS, ROWS = 40 * 2.0 ** -24, 84 * 2.0 ** -24


@pytest.mark.parametrize("H,P,N,G", [(4, 64, 16, 1), (2, 40, 24, 1), (2, 20, 100, 1), (1, 16, 4, 1), (1, 8, 200, 1), (2, 16, 64, 2)])
@pytest.mark.parametrize("rows", [700, 8000])
@pytest.mark.parametrize("kind", ["same", "same step", "any"])
def test_errors_do_not_grow_with_the_rows(hs, H, P, N, G, rows, kind):
    """Decays next to one, row after row: what rounding leaves out of them and of the state must not add up."""
    a = Layer(H, P, N, G, [rows, 3], dtype=torch.float32, step=-8.5, seed=56)
    if kind == "same":
        a.rows[:] = a.rows[0].clone()
    elif kind == "same step":
        a.rows[:, -H:] = a.rows[0, -H:].clone()
    y, _, ssm = a.reference()
    sy, _, ss = a.reference(sizes=True)
    a.run(hs)
    torch.cuda.synchronize()
    off, far = np.abs(_wide(a.ssm) - ssm)[a.slots.cpu().numpy()], np.abs(_wide(a.y) - y)
    assert (off <= STATE_ROWS * ss[a.slots.cpu().numpy()]).all(), (off / ss[a.slots.cpu().numpy()]).max()
    assert (far <= ROWS * sy).all(), (far / sy).max()


@pytest.mark.parametrize("shape", [(2, 64, 128, 1), (1, 130, 100, 1), (2, 8, 256, 1), (2, 20, 110, 2), (4, 64, 16, 1), (2, 20, 4, 1)])
@pytest.mark.parametrize("new", [[40] + [0] * 60, [1] * 30 + [20] + [0] * 40, [0] * 300 + [500, 1, 8, 9], [8, 9, 0, 0, 0, 0, 0, 0, 0]])
def test_requests_with_many_rows_among_empty_ones(hs, shape, new):
    """Hardly more rows than requests, and most of them one request's."""
    a = Layer(*shape, new, dtype=torch.float32, pad=2, seed=58)
    n = len(new)
    a.check(hs, fresh=(torch.arange(n, device="cuda") % 3 == 0).int(), keep=torch.tensor([x - x // 3 for x in new], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("shape", [(2, 64, 128, 1), (2, 40, 24, 1), (2, 16, 100, 1), (1, 8, 4, 1)])
@pytest.mark.parametrize("new", [[1], [6], [40], [200]])
def test_an_infinite_state_is_no_number_in_its_own_channel_alone(hs, shape, new):
    a, b = (Layer(*shape, new, dtype=torch.float32, seed=57) for _ in range(2))
    own = int(a.slots[0])
    a.ssm[own, 0, 3, 2], a.ssm[own, 0, 5, 1] = float("inf"), -float("inf")
    a.run(hs)
    torch.cuda.synchronize()
    got, want, size = _wide(a.ssm)[own], b.reference()[2][own], b.reference(sizes=True)[2][own]
    at = np.zeros(got.shape, bool)
    at[0, 3, 2] = at[0, 5, 1] = True
    assert not np.isfinite(got[at]).any() and _near(got, want, size)[~at].all()
    y, want, size = _wide(a.y), b.reference()[0], b.reference(sizes=True)[0]
    assert not np.isfinite(y[:, [3, 5]]).any() and np.delete(_near(y, want, size, HALF[torch.float32]), [3, 5], axis=1).all()


# Outputs of 32 bits, in the 2-norm over a call, where signs are any and errors add as squares: in roundings of 32 bits some 4 for each of x, B and C, 6 for the
# weights (exponential, logarithm, step, C . B), 4 for the gate, 2 each for what three bf16 parts leave and for the sums: below 12.  (Two parts leave 2^-18 of a
# factor: 4.6e-6, 77 of them.)  What a long request adds to its state by products takes two parts whatever its outputs are: the second part is 2^-8 of the value
# at most and 0.42 x 2^-8 in the mean square, its rounding as much of itself, so 0.18 x 2^-16 for either factor and for the product of two seconds that is left
# out: 0.31 x 2^-16 together, and 0.75 x 2^-16 is allowed.
DIGITS, TWO_PARTS = 16 * 2.0 ** -24, 3 * 2.0 ** -18


@pytest.mark.parametrize("shape", [(4, 64, 128, 2), (2, 64, 128, 1), (2, 40, 24, 1), (4, 64, 16, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("new", [[17] * 5, [32, 3, 9], [200], [700, 20, 1, 130], [3000], [1] * 9])
def test_outputs_of_32_bits_have_their_digits(hs, shape, dtype, new):
    a = Layer(*shape, new, dtype=dtype, out=torch.float32, pad=1, seed=59)
    y, _, ssm = a.reference()
    a.run(hs)
    torch.cuda.synchronize()
    off = np.linalg.norm(_wide(a.y)[:a.T] - y) / np.linalg.norm(y)
    own = a.slots.cpu().numpy()
    left = np.linalg.norm(_wide(a.ssm)[own] - ssm[own]) / np.linalg.norm(ssm[own])
    by_products = shape[1:3] == (64, 128) and max(new) > 32
    assert off <= DIGITS and left <= (TWO_PARTS if by_products else DIGITS), (off, left)


@pytest.mark.parametrize("lead,pitch", [(0, 0), (3, 5)])
@pytest.mark.parametrize("K", [2, 4])
def test_outputs_of_32_bits_of_rows_at_any_address(hs, lead, pitch, K):
    for dtype in (torch.bfloat16, torch.float32):
        a = Layer(2, 64, 128, 1, [3, 200, 20, 129], dtype=dtype, out=torch.float32, K=K, seed=60, lead=lead)
        buf = torch.full((a.rows_n, a.Di + pitch), 7.0, device="cuda")
        a.y = buf[:, pitch // 2:pitch // 2 + a.Di]
        n = torch.tensor([3, 77, 0, 128], dtype=torch.int32, device="cuda")
        a.check(hs, keep=n)
        assert (buf[:, :pitch // 2] == 7.0).all() and (buf[:, pitch // 2 + a.Di:] == 7.0).all()


@pytest.mark.parametrize("places,at", [(256, 0), (256, 100), (1000, 999)])
def test_a_piece_among_empty_places_goes_the_way_of_a_piece_alone(hs, places, at):
    """By products, to the bit, whatever the number of places without rows beside it; and so do what it commits and the tokens beside it."""
    alone = Layer(2, 64, 128, 1, [500], seed=61)
    among = Layer(2, 64, 128, 1, [0] * at + [500] + [0] * (places - 1 - at), seed=62)
    for name in ("cw", "cb", "bias", "A_log", "D"):
        setattr(among, name, getattr(alone, name))
    among.rows.copy_(alone.rows)
    own, there = int(alone.slots[0]), int(among.slots[at])
    among.conv[there], among.ssm[there] = alone.conv[own], alone.ssm[own]
    keep = torch.full((places,), 333, dtype=torch.int32, device="cuda")
    for y in ("own", None):
        alone.run(hs, y=y, keep=keep[:1])
        among.run(hs, y=y, keep=keep)
        torch.cuda.synchronize()
        assert torch.equal(alone.y, among.y) and torch.equal(alone.ssm[own], among.ssm[there]) and torch.equal(alone.conv[own], among.conv[there])


@pytest.mark.parametrize("new", [[0] * 200 + [300, 33, 32, 31, 9, 8, 1], [1] * 300 + [40] + [0] * 100 + [1] * 5])
def test_long_requests_among_tokens_and_empty_places(hs, new):
    for dtype, out in ((torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)):
        n = len(new)
        keep = torch.tensor([max(x - 3, 0) for x in new], dtype=torch.int32, device="cuda")
        fresh = (torch.arange(n, device="cuda") % 4 == 1).int()
        Layer(2, 64, 128, 1, new, dtype=dtype, out=out, pad=2, seed=63).check(hs, keep=keep, fresh=fresh)
        a = Layer(2, 64, 128, 1, new, dtype=dtype, out=out, seed=64)
        _, conv, ssm = a.reference(keep=keep, fresh=fresh)
        size = a.reference(sizes=True, keep=keep, fresh=fresh)[2]
        a.run(hs, y=None, keep=keep, fresh=fresh)
        np.testing.assert_array_equal(_wide(a.conv), conv)
        assert _near(_wide(a.ssm), ssm, size).all()


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K", [4, 2])
@pytest.mark.parametrize("new", [[31], [32], [33], [127], [128], [129], [256], [257, 0, 3], [1000], [9] * 12, [300, 32, 140, 1, 5]])
def test_outputs_of_16_bits_at_all_lengths(hs, new, K, out):
    for dtype, keep in ((torch.float32, None), (out, [x - x // 3 for x in new]), (torch.float32, [x // 2 + 1 for x in new])):
        a = Layer(2, 64, 128, 1, new, dtype=dtype, out=out, K=K, pad=1, seed=65)
        a.check(hs, **({} if keep is None else dict(keep=torch.tensor(keep, dtype=torch.int32, device="cuda"))))
