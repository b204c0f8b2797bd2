"""fp64 oracle of the rollout side: the append to a paged cache, the chunk's attention over it, the verification of
drafted tokens and the subtree ends of packed trees.  Plain loops over sequences, tokens and heads."""
from __future__ import annotations

import numpy as np


def tree_ends(pos_off, parent):
    """end[j]: the local position behind the last one that has j on its root path."""
    end = np.zeros(len(parent), np.int64)
    for o, e in zip(pos_off[:-1], pos_off[1:]):
        for i in range(o, e):
            j = i
            while j >= 0:
                end[j] = max(end[j], i - o + 1)
                j = parent[j]
    return end


def slots(kv_len, cu_new):
    """(sequence, slot) of every new token."""
    out = []
    for b, n in enumerate(np.diff(cu_new)):
        out += [(b, int(kv_len[b] - n + i)) for i in range(n)]
    return out


def _norm(x, w, eps):
    return x if w is None else x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * w


def _rotate(x, angle, style):
    """x [heads, D], angle [rot / 2]; also the size of what each output element adds up."""
    rot = 2 * len(angle)
    y, mag = x.copy(), np.abs(x)
    if rot:
        c, s = np.cos(angle), np.sin(angle)
        ia, ib = (np.arange(rot // 2), np.arange(rot // 2, rot)) if style == "half" else (np.arange(0, rot, 2), np.arange(1, rot, 2))
        a, b = x[:, ia], x[:, ib]
        y[:, ia], y[:, ib] = a * c - b * s, b * c + a * s
        mag[:, ia] = mag[:, ib] = np.abs(a) + np.abs(b)
    return y, mag


def kv_append(k_pages, v_pages, page_table, kv_len, cu_new, q, k, v, freq=None, positions=None, q_norm=None, k_norm=None,
              norm_eps=1e-6, rot_style="half"):
    """Updated copies of the pools, the queries of the rows in use, and the error scales of queries and pools."""
    kp, vp, out = k_pages.copy(), v_pages.copy(), q.copy()
    kmag, qmag = np.abs(kp), np.abs(q)
    ps = kp.shape[2]
    freq = np.zeros(0) if freq is None else freq
    for t, (b, slot) in enumerate(slots(kv_len, cu_new)):
        ang = (slot if positions is None else int(positions[t])) * freq
        out[t], qmag[t] = _rotate(_norm(q[t], q_norm, norm_eps), ang, rot_style)
        page = page_table[b, slot // ps]
        kp[page, :, slot % ps], kmag[page, :, slot % ps] = _rotate(_norm(k[t], k_norm, norm_eps), ang, rot_style)
        vp[page, :, slot % ps] = v[t]
    return dict(q=out, k_pages=kp, v_pages=vp, q_mag=qmag, k_mag=kmag)


def kv_attention(q, k_pages, v_pages, page_table, kv_len, cu_new, scale, slot_end=None):
    """out, lse, and per row and head: sum of p |v| (per element), largest |score|, largest sum of |q k| scale."""
    T, H, D = q.shape
    K, ps = k_pages.shape[1], k_pages.shape[2]
    out, pv = np.zeros((T, H, D)), np.zeros((T, H, D))
    lse, top, mag = np.full((T, H), -np.inf), np.zeros((T, H)), np.zeros((T, H))
    for t, (b, slot) in enumerate(slots(kv_len, cu_new)):
        j = np.arange(slot + 1)
        if slot_end is not None:
            j = j[slot < slot_end[b, :slot + 1]]
        if len(j) == 0:
            continue
        page = page_table[b, j // ps]
        for h in range(H):
            kk, vv = k_pages[page, h // (H // K), j % ps], v_pages[page, h // (H // K), j % ps]
            x = kk @ q[t, h] * scale
            m = x.max()
            e = np.exp(x - m)
            z = e.sum()
            lse[t, h] = m + np.log(z)
            out[t, h], pv[t, h] = (e / z) @ vv, (e / z) @ np.abs(vv)
            top[t, h], mag[t, h] = np.abs(x).max(), (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale)
    return dict(out=out, lse=lse, pv=pv, top=top, mag=mag)


def _log_softmax(z, tau):
    x = z / tau
    x = x - x.max()
    return x - np.log(np.exp(x).sum())


def draft_verify(logits, draft, cu_draft, u_accept, u_sample, draft_logits=None, temperature=1.0):
    B = len(cu_draft) - 1
    tokens, logp = np.full(len(logits), -1, np.int64), np.zeros(len(logits))
    accepted = np.zeros(B, np.int64)
    for b in range(B):
        d0, n = cu_draft[b], cu_draft[b + 1] - cu_draft[b]
        r0 = d0 + b
        for i in range(n + 1):
            lp = _log_softmax(logits[r0 + i], temperature)
            mass = np.exp(lp)
            if i < n:
                y = draft[d0 + i]
                q = np.zeros(len(lp))
                if draft_logits is None:
                    q[y] = 1.0
                else:
                    q = np.exp(_log_softmax(draft_logits[d0 + i], temperature))
                if float(u_accept[d0 + i]) * q[y] < mass[y]:
                    tokens[r0 + i], logp[r0 + i] = y, lp[y]
                    accepted[b] += 1
                    continue
                left = np.maximum(mass - q, 0.0)
                mass = left if left.sum() > 0 else mass  # nothing left over: drawn from p
            cum = np.cumsum(mass)
            y = int(np.searchsorted(cum, float(u_sample[b]) * cum[-1], side="right"))
            tokens[r0 + i], logp[r0 + i] = y, lp[y]
            break
    return dict(tokens=tokens, n_accepted=accepted, logp=logp)
