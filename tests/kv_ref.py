"""The paged 4-bit cache in plain numpy, written from the definitions in include/aasd.h: page
books as lists, values in 64 bits.  Only the quantiser is in 32 bits, because the definition
fixes each of its roundings."""
from __future__ import annotations

import numpy as np
import torch

PAGE = 64
NONE = -1
TINY = np.float32(2.0 ** -60)


def bf16(x):
    """float32 -> nearest bfloat16, as float32."""
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def head_bytes(D):
    return PAGE * D + 2 * PAGE * 4


def quantise(x):
    """float32 [..., D] -> codes, scale, minimum."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(x).all(-1)
        x = np.where(bad[..., None], np.float32(0), x)
        m = bf16(x.min(-1))
        s = bf16((x.max(-1) - m) * np.float32(1.0 / 15.0))
        s = np.maximum(s, TINY)
        inv = (np.float32(1.0) / s).astype(np.float32)
        c = np.clip(np.rint((x - m[..., None]) * inv[..., None]), 0, 15).astype(np.uint8)
    c = np.where(bad[..., None], np.uint8(0), c)
    m = np.where(bad, np.float32(0), m)
    s = np.where(bad, TINY, s)
    return c, s, m, bad


class Entry:
    """Codes, scale and minimum of one token's keys and values of all heads."""

    def __init__(self, k, v):
        self.k, self.v = quantise(k), quantise(v)

    def values(self, which):
        c, s, m, _ = self.k if which == "k" else self.v
        return s[..., None].astype(np.float64) * c + m[..., None].astype(np.float64)


def store(pages, slot, entry, D):
    """Puts an entry into uint8 pages [n, hkv, bytes]."""
    page, off = slot // PAGE, slot % PAGE
    h, kb = D // 2, PAGE * D // 2
    for i, (c, s, m, _) in enumerate((entry.k, entry.v)):
        b = c[:, :h] | (c[:, h:] << 4)
        if i == 0:
            pages[page, :, off * h:(off + 1) * h] = b
        else:
            pages[page, :, kb + off:2 * kb + off:PAGE] = b
        word = (m.view(np.uint32) & 0xFFFF0000) | (s.view(np.uint32) >> 16)
        at = 2 * kb + i * PAGE * 4 + off * 4
        pages[page, :, at:at + 4] = word.astype("<u4").view(np.uint8).reshape(-1, 4)


def load(pages, slot, D):
    """float64 keys and values [hkv, D] at a slot, straight from the bytes."""
    page, off = slot // PAGE, slot % PAGE
    h, kb = D // 2, PAGE * D // 2
    out = []
    for i in range(2):
        b = pages[page, :, off * h:(off + 1) * h] if i == 0 else pages[page, :, kb + off:2 * kb + off:PAGE]
        at = 2 * kb + i * PAGE * 4 + off * 4
        word = np.ascontiguousarray(pages[page, :, at:at + 4]).view("<u4")[:, 0]
        s = (word << 16).astype(np.uint32).view(np.float32).astype(np.float64)
        m = (word & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)
        c = np.concatenate([b & 15, b >> 4], -1).astype(np.float64)
        out.append(s[:, None] * c + m[:, None])
    return out


def plan(cached, new, table, held, stack, max_pages, rows_per_seq, n_tokens, depth=None):
    """table: list of page lists; stack: list (top last).  Changes table, held and stack."""
    B = len(cached)
    need = [-(-(cached[b] + new[b]) // PAGE) for b in range(B)]
    for b in range(B):
        while held[b] > need[b]:                    # pages go back in order of place
            stack.append(table[b].pop(need[b]))
            held[b] -= 1
    kv, offs, full, asked, start = [], [0], False, 0, len(stack)
    for b in range(B):
        off = b * rows_per_seq if rows_per_seq else offs[-1]
        fits = need[b] <= max_pages and (rows_per_seq > 0 or off + new[b] <= n_tokens)
        want = max(0, need[b] - held[b]) if fits else 0
        asked += want
        ok = fits and (want == 0 or asked <= start)
        if ok:
            for _ in range(want):
                table[b].append(stack.pop())
                held[b] += 1
        full |= not ok
        kv.append(cached[b] + (new[b] if ok else 0))
        offs.append((b + 1) * rows_per_seq if rows_per_seq else off + new[b])
    slots, pos = np.full(n_tokens, NONE, np.int32), np.full(n_tokens, NONE, np.int32)
    for b in range(B):
        for i in range(kv[b] - cached[b]):
            c, t = cached[b] + i, offs[b] + i
            slots[t] = table[b][c // PAGE] * PAGE + c % PAGE
            pos[t] = cached[b] + (int(depth[t]) if depth is not None else i)
    return dict(kv_len=np.asarray(kv, np.int32), tok_offsets=np.asarray(offs, np.int32), slot_map=slots, positions=pos,
                full=full)


def norm_rotate(x, w, cs, rot, inter, eps):
    """float64 [H, D] heads of one token; cs: float64 [rot]."""
    y = np.asarray(x, np.float64)
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    y = y.copy()
    half = rot // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + half)
        p, q = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = p * cs[i] - q * cs[half + i], q * cs[i] + p * cs[half + i]
    return y


def attend(q, keys, vals, visible, scale):
    """One token's queries [Hq, D] over entries [n, Hkv, D]; visible: indices.  Returns the output,
    the lse and, per head, the largest sum of |q_d k_d| (what rounding errors are measured by)."""
    Hq, D = q.shape
    G = Hq // keys.shape[1] if keys.shape[1] else 1
    out, lse, size = np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros(Hq)
    if len(visible) == 0:
        return out, lse, size
    for h in range(Hq):
        k, v = keys[visible, h // G], vals[visible, h // G]
        s = k @ q[h].astype(np.float64) * scale
        m = s.max()
        e = np.exp(s - m)
        out[h] = e @ v / e.sum()
        lse[h] = m + np.log(e.sum())
        size[h] = (np.abs(k) @ np.abs(q[h].astype(np.float64))).max() * abs(scale)
    return out, lse, size


def path_of(node, parent):
    out = []
    while node >= 0:
        out.append(int(node))
        node = parent[node]
    return out[::-1]
