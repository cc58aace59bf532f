"""Pins of the oracle for recurrent layers and for the rules of logits (oracle/state_oracle.py), against loops and other forms."""
import math

import numpy as np
import pytest

from oracle import state_oracle as so


def _layer(rng, H, P, N, G, K, T, slots):
    Di, dx = H * P, H * P + 2 * G * N
    return dict(rows=rng.standard_normal((T, Di + dx + H)), conv_w=rng.uniform(-0.5, 0.5, (dx, K)), conv_b=rng.standard_normal(dx) * 0.1,
                dt_bias=rng.standard_normal(H) - 1.0, A_log=rng.uniform(0, 1, H), Dskip=rng.standard_normal(H),
                conv_state=rng.standard_normal((slots, K - 1, dx)), ssm_state=rng.standard_normal((slots, H, P, N)))


@pytest.mark.parametrize("K", [1, 2, 4])
def test_scan_against_python_loops(rng, K):
    H, P, N, G, T = 4, 2, 3, 2, 5
    a = _layer(rng, H, P, N, G, K, T, 2)
    y, conv, ssm = so.chunk_scan(cu_q=[0, T], slots=[1], **a)
    Di, dx = H * P, H * P + 2 * G * N
    silu = lambda v: v / (1 + math.exp(-v))
    line = [list(x) for x in a["conv_state"][1]] + [list(x[Di:Di + dx]) for x in a["rows"]]
    S = a["ssm_state"][1].tolist()
    for t in range(T):
        u = [silu(a["conv_b"][c] + sum(a["conv_w"][c][j] * line[t + j][c] for j in range(K))) for c in range(dx)]
        for h in range(H):
            g = h // (H // G)
            dt = math.log1p(math.exp(a["rows"][t][Di + dx + h] + a["dt_bias"][h]))
            for p in range(P):
                total = 0.0
                for n in range(N):
                    S[h][p][n] = math.exp(-dt * math.exp(a["A_log"][h])) * S[h][p][n] + dt * u[h * P + p] * u[Di + g * N + n]
                    total += S[h][p][n] * u[Di + G * N + g * N + n]
                want = (total + a["Dskip"][h] * u[h * P + p]) * silu(a["rows"][t][h * P + p])
                assert abs(y[t, h * P + p] - want) <= 1e-12 * max(1.0, abs(want))
    np.testing.assert_allclose(ssm[1], S, rtol=1e-12)
    np.testing.assert_array_equal(ssm[0], a["ssm_state"][0])
    if K > 1:
        np.testing.assert_array_equal(conv[1], line[T:])


def test_scan_against_the_unrolled_form(rng):
    H, P, N, G, K, T = 2, 3, 4, 1, 4, 6
    a = _layer(rng, H, P, N, G, K, T, 1)
    y, _, ssm = so.chunk_scan(cu_q=[0, T], **a)
    Di, dx = H * P, H * P + 2 * G * N
    raw = np.concatenate([a["conv_state"][0], a["rows"][:, Di:Di + dx]])
    u = np.stack([so.silu((raw[t:t + K].T * a["conv_w"]).sum(1) + a["conv_b"]) for t in range(T)])
    x, b, c = u[:, :Di].reshape(T, H, P), u[:, Di:Di + N], u[:, Di + N:]
    dt = np.log1p(np.exp(a["rows"][:, Di + dx:] + a["dt_bias"]))
    fall = np.cumsum(-dt * np.exp(a["A_log"]), axis=0)
    for h in range(H):
        w = np.tril(np.exp(fall[:, None, h] - fall[None, :, h]) * dt[None, :, h] * (c @ b.T))
        o = w @ x[:, h] + np.exp(fall[:, h])[:, None] * (c @ a["ssm_state"][0, h].T) + a["Dskip"][h] * x[:, h]
        np.testing.assert_allclose(y.reshape(T, H, P)[:, h], o * so.silu(a["rows"][:, :Di]).reshape(T, H, P)[:, h], rtol=1e-10)
        s = np.exp(fall[-1, h]) * a["ssm_state"][0, h] + np.einsum("tp,tn->pn", (np.exp(fall[-1, h] - fall[:, h]) * dt[:, h])[:, None] * x[:, h], b)
        np.testing.assert_allclose(ssm[0, h], s, rtol=1e-10)


def test_scan_in_pieces_and_of_kept_rows(rng):
    H, P, N, G, K, T = 2, 2, 3, 2, 4, 9
    a = _layer(rng, H, P, N, G, K, T, 3)
    whole = so.chunk_scan(cu_q=[0, T], slots=[2], fresh=[1], **a)
    conv, ssm, y = a["conv_state"], a["ssm_state"], []
    for lo, hi in ((0, 1), (1, 3), (3, 9)):
        part, conv, ssm = so.chunk_scan(cu_q=[0, hi - lo], slots=[2], fresh=[int(lo == 0)], **dict(a, rows=a["rows"][lo:hi], conv_state=conv, ssm_state=ssm))
        y.append(part)
    np.testing.assert_allclose(np.concatenate(y), whole[0], rtol=1e-12)
    np.testing.assert_allclose(ssm, whole[2], rtol=1e-12)
    np.testing.assert_array_equal(conv, whole[1])
    for keep in (0, 1, 2, 5):
        got = so.chunk_scan(cu_q=[0, T], slots=[1], keep=[keep - 1], keep_more=1, **a)
        less = so.chunk_scan(cu_q=[0, keep], slots=[1], **dict(a, rows=a["rows"][:keep]))
        np.testing.assert_array_equal(got[1], less[1])
        np.testing.assert_array_equal(got[2], less[2])


def test_scan_without_a_place(rng):
    a = _layer(rng, 2, 2, 3, 1, 3, 4, 2)
    y, conv, ssm = so.chunk_scan(cu_q=[0, 4], slots=[-1], **a)
    np.testing.assert_array_equal(y, so.chunk_scan(cu_q=[0, 4], slots=[0], fresh=[1], **a)[0])
    np.testing.assert_array_equal(ssm, a["ssm_state"])
    zeros = so.chunk_scan(cu_q=[0, 0], slots=[1], fresh=[1], **a)
    assert not zeros[1][1].any() and not zeros[2][1].any() and (zeros[2][0] == a["ssm_state"][0]).all()


def test_rules_against_python_loops(rng):
    V, cu = 40, [0, 3, 3, 4]
    z = rng.standard_normal((5, V)) * 3
    history, lens, first = rng.integers(0, V, (3, 12)), [12, 5, 0], [4, 5, 0]
    drafts = rng.integers(0, V, (3, 4))
    r, f, p = [1.3, 1.0, 0.7], [0.2, 0.1, -0.3], [0.5, 0.0, 0.4]
    ids, vals, counts = rng.integers(0, V, (3, 6)), rng.standard_normal((3, 6)), [6, 2, 0]
    ids[0, 1] = ids[0, 0]
    mask, rule = rng.integers(-2 ** 31, 2 ** 31, (2, 2)).astype(np.int32), [1, -1, 0, 1, 0]
    got = so.adjust_logits(z, cu, history, lens, first, drafts, r, f, p, ids, vals, counts, mask, rule)
    for b in range(3):
        for i in range(cu[b + 1] - cu[b]):
            t = cu[b] + i
            answer = list(history[b][first[b]:lens[b]]) + list(drafts[b][:i])
            for v in range(V):
                x, n = z[t, v], answer.count(v)
                if n or v in history[b][:first[b]]:
                    x = x / r[b] if x > 0 else x * r[b]
                if n:
                    x = x - f[b] * n - p[b]
                x += sum(vals[b][j] for j in range(counts[b]) if ids[b][j] == v)
                if rule[t] >= 0 and not (int(mask[rule[t]][v // 32]) >> (v % 32)) & 1:
                    x = -math.inf
                assert got[t, v] == pytest.approx(x, rel=1e-12)
    np.testing.assert_array_equal(got[4], z[4])
    np.testing.assert_array_equal(so.adjust_logits(z), z)
    np.testing.assert_array_equal(so.adjust_logits(z, history=history[:, :0].repeat(2, 0)[:5], repetition=[9.0] * 5), z)
