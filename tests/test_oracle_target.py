"""Pins of the oracle for the target's side of an iteration (oracle/target_oracle.py), against loops and closed forms."""
import numpy as np
import pytest

from oracle import target_oracle as to


def test_rope_keeps_lengths_and_position_zero(rng):
    x = rng.standard_normal((5, 3, 32))
    axis = [j % 3 for j in range(16)]
    np.testing.assert_allclose(to.chunk_rope(x, np.zeros((3, 5)), axis, 1e4), x, rtol=0, atol=1e-15)
    y = to.chunk_rope(x, rng.integers(0, 10 ** 6, (3, 5)), axis, 1e4)
    np.testing.assert_allclose(y[..., :16] ** 2 + y[..., 16:] ** 2, x[..., :16] ** 2 + x[..., 16:] ** 2, rtol=1e-12)


def test_rope_of_equal_axes_is_the_rope_of_one(rng):
    x, p = rng.standard_normal((7, 2, 64)), rng.integers(0, 5000, 7)
    one = to.chunk_rope(x, p[None], [0] * 32, 1e6)
    np.testing.assert_array_equal(to.chunk_rope(x, np.stack([p, p, p]), [0] * 8 + [1] * 12 + [2] * 12, 1e6), one)
    # and that of the first pair is the rotation by the position itself
    c, s = np.cos(p)[:, None], np.sin(p)[:, None]
    np.testing.assert_allclose(one[..., 0], x[..., 0] * c - x[..., 32] * s, atol=1e-12)


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_rope_products_depend_on_distances_along_every_axis(rng, axis):
    a, b = rng.standard_normal((2, 1, 1, 24))
    axes = [j % 3 for j in range(8)]                       # 16 of 24 values turn
    p, d = rng.integers(0, 900, 3), rng.integers(0, 50, 3)
    base = to.chunk_rope(a, p[:, None], axes, 1e4) @ np.swapaxes(to.chunk_rope(b, (p + d)[:, None], axes, 1e4), 1, 2)
    q = p.copy()
    q[axis] += 333
    moved = to.chunk_rope(a, q[:, None], axes, 1e4) @ np.swapaxes(to.chunk_rope(b, (q + d)[:, None], axes, 1e4), 1, 2)
    np.testing.assert_allclose(moved, base, rtol=1e-10)


def _cache(rng, B, page=4, width=6, Hkv=2, dh=8):
    pages = B * width + 1
    table = rng.permutation(pages)[:B * width].reshape(B, width)
    return rng.standard_normal((pages, page, Hkv, dh)), rng.standard_normal((pages, page, Hkv, dh)), table


@pytest.mark.parametrize("window", [0, 1, 5])
def test_attention_against_loops(rng, window):
    K, V, table = _cache(rng, 3)
    cu, kv = [0, 4, 4, 7], [11, 9, 3]
    q = rng.standard_normal((7, 4, 8))
    got = to.chunk_attention(q, K, V, table, cu, kv, window=window)
    t = 0
    for b in range(3):
        n = cu[b + 1] - cu[b]
        for i in range(n):
            p = kv[b] - n + i
            for h in range(4):
                num, den = np.zeros(8), 0.0
                for j in range(p + 1):
                    if window and j <= p - window:
                        continue
                    k, v = K[table[b, j // 4], j % 4, h // 2], V[table[b, j // 4], j % 4, h // 2]
                    w = np.exp(float(q[t, h] @ k) / np.sqrt(8))
                    num, den = num + w * v, den + w
                np.testing.assert_allclose(got[t, h], num / den, rtol=1e-12)
            t += 1
    if window == 1:
        np.testing.assert_allclose(got[0, 0], V[table[0, 7 // 4], 7 % 4, 0], rtol=1e-14)


def test_attention_in_pieces_and_rows_that_see_nothing(rng):
    K, V, table = _cache(rng, 1)
    q = rng.standard_normal((9, 2, 8))
    whole = to.chunk_attention(q, K, V, table, [0, 9], [15])
    parts = [to.chunk_attention(q[i:i + 1], K, V, table, [0, 1], [7 + i]) for i in range(9)]
    np.testing.assert_allclose(whole, np.concatenate(parts), rtol=1e-13)
    short = to.chunk_attention(q, K, V, table, [0, 9], [4])            # more rows than cached tokens
    assert (short[:5] == 0).all() and (short[5:] != 0).any()


@pytest.mark.parametrize("sampled", [True, False])
def test_verify_emits_the_targets_distribution(rng, sampled):
    """Over all (draft, alpha, u) the first emitted token has the target's distribution: drafts by their own probability, the two
    uniform numbers on a grid."""
    V, N = 5, 400
    z, d = rng.standard_normal((2, 1, V)) * 1.5
    p = np.exp(z[0]) / np.exp(z[0]).sum()
    q = np.exp(d[0]) / np.exp(d[0]).sum()
    share = np.zeros(V)
    grid = (np.arange(N) + 0.5) / N
    target = np.concatenate([z, z])
    for x in (range(V) if sampled else [int(np.argmax(d))]):
        ids = np.full((N, 1), x)
        n, tok = to.verify(np.tile(target, (N, 1)), np.tile(d[None], (N, 1, 1)) if sampled else None, ids, grid[:, None], np.zeros(N))
        stands = n.mean()
        # (u only moves the token behind: taken on the grid for a refused draft)
        _, tok = to.verify(np.tile(target, (N, 1)), np.tile(d[None], (N, 1, 1)) if sampled else None, ids, np.ones((N, 1)), grid)
        behind = np.bincount(tok[tok[:, 1] == -1][:, 0], minlength=V) / N
        weight = q[x] if sampled else 1.0
        share[x] += weight * stands
        if stands < 1:
            share += weight * (1 - stands) * behind
    np.testing.assert_allclose(share, p, atol=6.0 / N)


def test_verify_greedy_and_equal_models(rng):
    B, k, V = 3, 4, 30
    z = rng.standard_normal((B * (k + 1), V))
    top = z.argmax(1).reshape(B, k + 1)
    ids = top[:, :k].copy()
    ids[1, 2] = (ids[1, 2] + 1) % V
    n, tok = to.verify(z, None, ids, rng.random((B, k)), rng.random(B), temperature=np.zeros(B))
    assert n.tolist() == [4, 2, 4]
    assert tok[0].tolist() == top[0].tolist() and tok[1].tolist() == top[1, :3].tolist() + [-1, -1]
    # a drafter that is the target: everything stands
    draft = z.reshape(B, k + 1, V)[:, :k]
    n, _ = to.verify(z, draft, rng.integers(0, V, (B, k)), np.full((B, k), 1.0), rng.random(B))
    assert (n == k).all()
    # ragged rows: none at all, the token alone
    n, tok = to.verify(z, draft, ids, rng.random((B, k)), rng.random(B), cu_q=[0, 0, 1, 3])
    assert tok[0].tolist() == [-1] * 5 and n[1] == 0 and tok[1, 0] >= 0 and (tok[1, 1:] == -1).all()


def test_verify_pruned_vocabulary_and_masks(rng):
    V, keep = 12, np.array([1, 4, 5, 9])
    z = rng.standard_normal((2, V))
    d = np.full((1, 1, 4), -np.inf)
    d[0, 0, 2] = 0.0                                       # all of q on token 5
    n, tok = to.verify(z, d, np.array([[5]]), np.array([[1.0]]), np.array([0.999999]), vocab_map=keep)
    p = np.exp(z[0]) / np.exp(z[0]).sum()
    assert n[0] == 0 and tok[0, 0] != 5 and tok[0, 1] == -1 and p[tok[0, 0]] > 0
    z[0, 5] = np.nan                                       # a token without weight never stands, even at alpha 0
    n, _ = to.verify(z, d, np.array([[5]]), np.array([[0.0]]), np.array([0.5]), vocab_map=keep)
    assert n[0] == 0
    z[:] = -np.inf
    n, tok = to.verify(z, d, np.array([[5]]), np.array([[0.0]]), np.array([0.5]), vocab_map=keep)
    assert n[0] == 0 and tok[0, 0] == 0
