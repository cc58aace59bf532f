"""What the scan of a chunk and the rules of logits refuse, on the host and before anything is enqueued (no GPU needed): the C entry points with made-up
addresses, and the binding's own checks."""
import pytest
import torch

import paper_2609_24197_b200 as hs
from paper_2609_24197_b200 import build as hbuild

A = 1 << 20                     # an address that is never followed
BF16, F32, I32, F16 = hs.HSPEC_BF16, hs.HSPEC_F32, hs.HSPEC_I32, hs.HSPEC_F16


@pytest.fixture(scope="module")
def lib():
    hbuild.build()
    return hs.load_library()


def _scan(lib, **over):
    a = dict(x=A, in_dtype=BF16, ld=2 * 512 + 2 * 128 + 8, dt=None, cw=A, cb=A, bias=A, A_log=A, D=A, cu=A, B=4, slots=A, fresh=A, keep=A, more=0, conv=A, ssm=A,
             n_slots=8, y=A, y_dtype=BF16, ldy=512, T=10, Di=512, P=64, N=128, G=1, K=4, ws=A, ws_bytes=1 << 40)
    a.update(over)
    return lib.hspec_op_chunk_scan(*a.values(), None), lib.hspec_last_error(None).decode()


@pytest.mark.parametrize("over,code,text", [
    (dict(x=None), -1, "bad argument"), (dict(cw=None), -1, "bad argument"), (dict(A_log=None), -1, "bad argument"), (dict(cu=None), -1, "bad argument"),
    (dict(ssm=None), -1, "bad argument"), (dict(ws=None), -1, "bad argument"), (dict(B=0), -1, "bad argument"), (dict(T=-1), -1, "bad argument"),
    (dict(n_slots=0), -1, "bad argument"), (dict(in_dtype=I32), -1, "rows must be"), (dict(y_dtype=9), -1, "rows must be"),
    (dict(Di=500), -2, "fill Di"), (dict(G=3), -2, "fill Di"), (dict(P=0), -2, "fill Di"), (dict(N=257), -2, "256 state"), (dict(K=0), -2, "1 to 4"),
    (dict(K=5), -2, "1 to 4"), (dict(conv=None), -1, "carried rows"), (dict(ld=2 * 512 + 2 * 128 + 7), -1, "row pitch"), (dict(ldy=511), -1, "row pitch"),
    (dict(x=A + 1), -1, "misaligned"), (dict(conv=A + 1), -1, "misaligned"), (dict(y=A + 2, y_dtype=F32), -1, "misaligned"),
    (dict(ssm=A + 4), -1, "16-byte"), (dict(ws_bytes=100), -4, "workspace too small"), (dict(ws=A + 16), -1, "256-byte"), (dict(B=65536), -2, "65535"),
    (dict(Di=1 << 25, ld=1 << 28, ldy=1 << 25), -2, "2^24")])
def test_scan_refuses(lib, over, code, text):
    rc, msg = _scan(lib, **over)
    assert rc == code and "hspec_op_chunk_scan" in msg and text in msg


def test_scan_workspace_grows_with_rows_and_requests(lib):
    size = hs.hspec_chunk_scan_workspace_bytes
    assert size(10, 4, 500, 64, 128, 1) == 0 and size(-1, 4, 512, 64, 128, 1) == 0 and size(10, 0, 512, 64, 128, 1) == 0
    for shape in ((512, 64, 128, 1), (8192, 64, 128, 4), (512, 64, 16, 1), (960, 40, 24, 3)):
        last = 0
        for T in (0, 1, 5, 32, 33, 64, 128, 200, 1000, 8192, 30000):
            row = [size(T, B, *shape) for B in (1, 2, 7, 31, 64, 300, 5000)]
            assert row == sorted(row) and row[0] >= last, (T, shape)
            last = row[0]


def _rules(lib, **over):
    a = dict(z=A, in_dtype=BF16, ld=1000, out=2 * A, out_dtype=F32, ldo=1000, T=12, V=1000, cu=A, B=4, hist=A, stride=64, lens=A, prompt=A, drafts=A, k=4, rep=A,
             freq=A, pres=A, ids=A, vals=A, counts=A, n=8, mask=A, masks=3, mstride=32, mrows=A)
    a.update(over)
    return lib.hspec_op_adjust_logits(*a.values(), None), lib.hspec_last_error(None).decode()


@pytest.mark.parametrize("over,code,text", [
    (dict(z=None), -1, "bad argument"), (dict(out=None), -1, "bad argument"), (dict(T=-1), -1, "bad argument"), (dict(V=0), -1, "bad argument"),
    (dict(B=0), -1, "bad argument"), (dict(ld=999), -1, "bad argument"), (dict(ldo=999), -1, "bad argument"), (dict(ids=None), -1, "bad argument"),
    (dict(vals=None), -1, "bad argument"), (dict(in_dtype=I32), -1, "logits must be"), (dict(out_dtype=F16), -1, "logits must be"),
    (dict(in_dtype=F32, out_dtype=BF16), -1, "logits must be"), (dict(z=A + 1), -1, "misaligned"), (dict(out=2 * A + 2), -1, "misaligned"),
    (dict(out=A), -1, "in place"), (dict(out=A, out_dtype=BF16, ldo=1001), -1, "in place"), (dict(cu=None), -1, "one row"), (dict(stride=0), -1, "too small"),
    (dict(k=0), -1, "too small"), (dict(n=0), -1, "too small"), (dict(masks=0), -1, "too small"), (dict(mstride=31), -1, "too small"),
    (dict(stride=1 << 20), -2, "2^20"), (dict(n=1025), -2, "1024 biases"), (dict(V=2 ** 31 - 1, ld=2 ** 31, ldo=2 ** 31, mstride=2 ** 27), -2, "2^30 tokens")])
def test_rules_refuse(lib, over, code, text):
    rc, msg = _rules(lib, **over)
    assert rc == code and "hspec_op_adjust_logits" in msg and text in msg


def test_no_rows_are_nothing_to_do(lib):
    assert _rules(lib, T=0, z=None, out=None)[0] == 0


def test_the_binding_refuses_before_the_library(lib):
    f = lambda *s: torch.zeros(s)
    ints = torch.zeros(3, dtype=torch.int32)
    layer = (f(20, 4), f(20), f(1), f(1), f(1))
    with pytest.raises(hs.HSpecError, match="current CUDA device"):
        hs.hspec_op_chunk_scan(f(5, 29), *layer, ints, f(2, 3, 20), f(2, 1, 8, 6), f(5, 8), torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(hs.HSpecError, match="channels are not those"):
        hs.hspec_op_chunk_scan(f(5, 29), *layer, ints, f(2, 3, 20), f(2, 1, 8, 7), f(5, 8), torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(hs.HSpecError, match="current CUDA device"):
        hs.hspec_op_adjust_logits(f(2, 9), f(2, 9))
