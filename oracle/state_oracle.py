"""CPU oracle for a hybrid target's recurrent layers and for the rules of its logits.  TEST INFRASTRUCTURE ONLY.

Plain numpy restatements in 64 bits, written from the definitions; shares no code with the CUDA library and is never imported by
the product path.

  chunk_scan      short causal convolution, selective scan and gate of a ragged chunk, token by token, with carried rows and states
  adjust_logits   penalties for repeated tokens, biases and allowed tokens, row by row of a drafted block

What pins each function (tests/test_oracle_state.py):
  chunk_scan      explicit Python loops over nested lists, the unrolled ("quadratic") form, pieces of a prompt equal the whole, kept rows
                  equal a shorter call
  adjust_logits   explicit Python loops over a dictionary of counts, no rule leaves the logits as they are
"""
import numpy as np


def silu(v):
    return v / (1.0 + np.exp(-v))


def chunk_scan(rows, conv_w, conv_b, dt_bias, A_log, Dskip, cu_q, conv_state, ssm_state, dt_raw=None, slots=None, fresh=None, keep=None, keep_more=0,
               sizes=False):
    """rows [T, z | x | B | C (| dt)], conv_state [slots, K - 1, d_xBC], ssm_state [slots, H, P, N] -> (y [cu_q[-1], Di], conv_state, ssm_state), new arrays.
    sizes: the sum of the absolute values of everything that enters a result, in its place (what rounding errors are relative to)."""
    n_slots, H, P, N = ssm_state.shape
    Di, (dx, K) = H * P, conv_w.shape
    G = (dx - Di) // (2 * N)
    w, b = np.asarray(conv_w, np.float64), np.asarray(conv_b, np.float64)
    conv, ssm = np.array(conv_state, np.float64), np.array(ssm_state, np.float64)
    y = np.zeros((int(cu_q[-1]), Di))
    A = -np.exp(np.asarray(A_log, np.float64))
    mag = np.abs if sizes else (lambda v: v)
    ssm = mag(ssm)
    for r in range(len(cu_q) - 1):
        lo, n = int(cu_q[r]), int(cu_q[r + 1]) - int(cu_q[r])
        slot = r if slots is None else int(slots[r])
        there = 0 <= slot < n_slots
        new = not there or (fresh is not None and bool(fresh[r]))
        kept = n if keep is None else min(max(int(keep[r]) + keep_more, 0), n)
        past = np.zeros((K - 1, dx)) if new else conv[slot].copy()
        S = np.zeros((H, P, N)) if new else ssm[slot].copy()
        raw = np.concatenate([past, np.asarray(rows[lo:lo + n, Di:Di + dx], np.float64)])
        at = [S.copy()]
        for t in range(n):
            if sizes:
                u = 1.1 * (np.sum(np.abs(raw[t:t + K].T * w), axis=1) + np.abs(b))           # (the convolution's terms; SiLU's slope is below 1.1)
            else:
                u = silu(np.sum(raw[t:t + K].T * w, axis=1) + b)
            x = u[:Di].reshape(H, P)
            k, q = (np.repeat(u[Di + i * G * N:Di + (i + 1) * G * N].reshape(G, N), H // G, axis=0) for i in (0, 1))
            d = np.asarray(rows[lo + t, Di + dx:] if dt_raw is None else dt_raw[lo + t], np.float64)
            dt = np.logaddexp(d + np.asarray(dt_bias, np.float64), 0.0)
            S = S * np.exp(dt * A)[:, None, None] + (dt[:, None] * x)[:, :, None] * k[:, None, :]
            out = np.einsum("hpn,hn->hp", S, q) + mag(np.asarray(Dskip, np.float64))[:, None] * x
            y[lo + t] = out.reshape(Di) * mag(silu(np.asarray(rows[lo + t, :Di], np.float64)))
            at.append(S.copy())
        if there and (kept > 0 or new):
            conv[slot] = raw[kept:kept + K - 1]
            ssm[slot] = at[kept]
    return y, conv, ssm


def adjust_logits(logits, cu_q=None, history=None, history_lens=None, prompt_lens=None, drafts=None, repetition=None, frequency=None, presence=None,
                  bias_ids=None, bias_values=None, bias_counts=None, mask=None, mask_rows=None):
    """logits [T, V] -> float64 [T, V]; rows behind cu_q[-1] as they are."""
    out = np.array(logits, np.float64)
    T, V = out.shape
    cu = list(range(T + 1)) if cu_q is None else [int(x) for x in cu_q]
    for r in range(len(cu) - 1):
        text, first = np.zeros(0, np.int64), 0
        if history is not None:
            n = history.shape[1] if history_lens is None else min(max(int(history_lens[r]), 0), history.shape[1])
            text = np.asarray(history[r, :n], np.int64)
            first = 0 if prompt_lens is None else min(max(int(prompt_lens[r]), 0), n)
        for i in range(cu[r + 1] - cu[r]):
            z = out[cu[r] + i]
            mine = text[first:]
            if drafts is not None:
                mine = np.concatenate([mine, np.asarray(drafts[r, :min(i, drafts.shape[1])], np.int64)])
            mine = mine[(mine >= 0) & (mine < V)]
            said = np.bincount(mine, minlength=V)
            prompt = text[:first]
            seen = (said > 0) | (np.bincount(prompt[(prompt >= 0) & (prompt < V)], minlength=V) > 0)
            if repetition is not None:
                rep = float(repetition[r])
                z[seen] = np.where(z[seen] > 0, z[seen] / rep, z[seen] * rep)
            on = said > 0
            if frequency is not None:
                z[on] -= float(frequency[r]) * said[on]
            if presence is not None:
                z[on] -= float(presence[r])
            if bias_ids is not None:
                n = bias_ids.shape[1] if bias_counts is None else min(max(int(bias_counts[r]), 0), bias_ids.shape[1])
                for v, x in zip(bias_ids[r, :n], bias_values[r, :n]):
                    if 0 <= v < V:
                        z[v] += float(x)
            m = -1 if mask is None else (cu[r] + i if mask_rows is None else int(mask_rows[cu[r] + i]))
            if mask is not None and 0 <= m < len(mask):
                word = np.asarray(mask[m]).astype(np.int64) & 0xffffffff
                v = np.arange(V)
                z[(word[v // 32] >> (v % 32)) & 1 == 0] = -np.inf
    return out
