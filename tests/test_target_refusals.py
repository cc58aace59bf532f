"""What the operators of the target's side refuse, on the host and before anything is enqueued (no GPU needed): the C entry points with made-up
addresses, and the binding's own checks."""
import ctypes as C

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


def _rope(lib, **over):
    a = dict(qkv=A, in_dtype=BF16, ld=48 * 128, pos=A, axes=3, pair_axis=bytes([0, 1, 2, 2] * 16), pairs=64, qw=A, kw=A, eps=1e-6, theta=1e6, cu=A, kv=A,
             B=4, table=A, stride=8, q=A, k=A, v=A, out=BF16, pages=100, T=10, Hq=32, Hkv=8, dh=128, page=16)
    a.update(over)
    return lib.hspec_op_chunk_rope_write(*a.values(), None), lib.hspec_last_error(None).decode()


@pytest.mark.parametrize("over,code,text", [
    (dict(qkv=None), -1, "bad argument"), (dict(cu=None), -1, "bad argument"), (dict(k=None), -1, "bad argument"), (dict(qw=None), -1, "bad argument"),
    (dict(theta=0.0), -1, "bad argument"), (dict(theta=float("nan")), -1, "bad argument"), (dict(eps=-1.0), -1, "bad argument"), (dict(in_dtype=I32), -1, "qkv must be"),
    (dict(out=F32), -2, "bf16 or fp16"), (dict(Hq=30), -2, "multiple of the KV heads"), (dict(Hkv=0), -2, "multiple"), (dict(dh=96), -2, "head dim"),
    (dict(q=A + 8), -2, "16-byte"), (dict(v=A + 2), -2, "16-byte"), (dict(pairs=4), -2, "rotated pairs"), (dict(pairs=72), -2, "rotated pairs"),
    (dict(pairs=60), -2, "rotated pairs"), (dict(axes=0), -1, "axes"), (dict(axes=9), -1, "axes"), (dict(pos=None), -1, "axes"),
    (dict(axes=2), -1, "pair_axis"), (dict(ld=48 * 128 - 1), -1, "row pitch"), (dict(B=0), -2, "bad argument"), (dict(page=0), -2, "bad argument"),
    (dict(stride=0), -2, "bad argument"), (dict(pages=0), -2, "bad argument"), (dict(pages=1 << 31), -2, "bad argument"), (dict(T=-1), -2, "bad argument")])
def test_rope_write_refuses(lib, over, code, text):
    rc, msg = _rope(lib, **over)
    assert rc == code and "hspec_op_chunk_rope_write" in msg and text in msg


def _attn(lib, **over):
    a = dict(q=A, ldq=32 * 128, k=A, v=A, pages=100, table=A, stride=8, cu=A, kv=A, B=4, o=A, ldo=32 * 128, dtype=BF16, T=10, Hq=32, Hkv=8, dh=128, page=16,
             window=0, scale=0.0, ws=A, ws_bytes=1 << 40)
    a.update(over)
    return lib.hspec_op_chunk_attention(*a.values(), None), lib.hspec_last_error(None).decode()


@pytest.mark.parametrize("over,code,text", [
    (dict(q=None), -1, "bad argument"), (dict(o=None), -1, "bad argument"), (dict(ws=None), -1, "bad argument"), (dict(window=-1), -1, "bad argument"),
    (dict(scale=-0.5), -1, "bad argument"), (dict(scale=float("nan")), -1, "bad argument"), (dict(scale=float("inf")), -1, "bad argument"),
    (dict(dtype=F32), -2, "bf16 or fp16"), (dict(dh=256), -2, "head dim"), (dict(Hq=33), -2, "multiple"), (dict(k=A + 4), -2, "16-byte"),
    (dict(ldq=32 * 128 - 8), -1, "rows of q and o"), (dict(ldo=32 * 128 + 4), -1, "rows of q and o"), (dict(o=A + 8), -1, "rows of q and o"),
    (dict(ws_bytes=0), -4, "workspace too small"), (dict(ws=A + 16), -1, "256-byte"), (dict(B=0), -2, "bad argument"),
    (dict(B=8193), -2, "8192 requests"), (dict(T=2 ** 27), -2, "too many rows"), (dict(Hq=513, Hkv=1, ldq=513 * 128, ldo=513 * 128), -2, "512 query heads")])
def test_chunk_attention_refuses(lib, over, code, text):
    rc, msg = _attn(lib, **over)
    assert rc == code and "hspec_op_chunk_attention" in msg and text in msg


def _verify(lib, **over):
    a = dict(target=A, t_dtype=F32, ld_t=1000, T=68, draft=A, d_dtype=F32, ld_d=1000, ids=A, cu=None, vmap=None, temp=None, alpha=A, u=A, n=A, tok=A, B=4, k=16,
             V=1000, Vd=1000, ws=A, ws_bytes=1 << 30)
    a.update(over)
    return lib.hspec_op_verify(*a.values(), None), lib.hspec_last_error(None).decode()


@pytest.mark.parametrize("over,code,text", [
    (dict(target=None), -1, "bad argument"), (dict(u=None), -1, "bad argument"), (dict(k=0), -1, "bad argument"), (dict(ld_t=999), -1, "bad argument"),
    (dict(t_dtype=I32), -1, "logits must be"), (dict(d_dtype=9), -1, "logits must be"), (dict(T=67), -1, "k + 1 rows"), (dict(Vd=900), -1, "needs its map"),
    (dict(Vd=0, vmap=A), -1, "drafter vocabulary"), (dict(Vd=1001, vmap=A), -1, "drafter vocabulary"), (dict(ld_d=999), -1, "drafter vocabulary"),
    (dict(B=1 << 24, k=1 << 5, cu=A), -2, "too many drafts"), (dict(V=2 ** 31 - 1, Vd=2 ** 31 - 1, ld_t=2 ** 31, ld_d=2 ** 31), -2, "2^30 tokens"),
    (dict(ws_bytes=100), -4, "workspace too small"), (dict(ws=A + 4), -1, "256-byte")])
def test_verify_refuses(lib, over, code, text):
    rc, msg = _verify(lib, **over)
    assert rc == code and "hspec_op_verify" in msg and text in msg


def test_an_empty_chunk_is_nothing_to_do(lib):
    assert _rope(lib, T=0, qkv=None, q=None)[0] == 0
    assert _attn(lib, T=0, q=None, o=None)[0] == 0


def test_workspaces(lib):
    assert hs.hspec_verify_workspace_bytes(0, 4) == 0 and hs.hspec_verify_workspace_bytes(3, 16) >= 3 * 16 * 16
    assert hs.hspec_chunk_attention_workspace_bytes(32, 8, 128) > 0


def test_the_binding_refuses_before_the_library(lib):
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    pool, ints = torch.zeros((5, 16, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(hs.HSpecError, match="current CUDA device"):
        hs.hspec_op_chunk_attention(q, pool, pool, ints[None], ints, ints[:1], q.clone(), torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(hs.HSpecError, match="current CUDA device"):
        hs.hspec_op_verify(torch.zeros((4, 9)), None, torch.zeros((1, 3), dtype=torch.int32), torch.zeros((1, 3)), torch.zeros(1), ints[:1],
                           torch.zeros((1, 4), dtype=torch.int32), torch.zeros(8, dtype=torch.uint8))


def test_verify_without_rows_needs_their_offsets(lib):
    for over, text in ((dict(T=0), "k + 1 rows"), (dict(T=0, target=None), "k + 1 rows"), (dict(T=-1, cu=A), "bad argument"), (dict(T=1, target=None, cu=A), "bad argument")):
        rc, msg = _verify(lib, **over)
        assert rc == -1 and "hspec_op_verify" in msg and text in msg


def test_a_scale_whose_product_with_log2_e_is_infinite(lib):
    for scale in (2.36e38, 3.0e38):
        rc, msg = _attn(lib, scale=scale)
        assert rc == -1 and "hspec_op_chunk_attention" in msg and "bad argument" in msg
