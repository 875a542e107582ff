"""Batches for language models that read images and video, from their definitions, in 64 bits or more: patch rows,
places of tokens on three axes, rotary embedding, slots in a paged cache.  Plain numpy; test infrastructure only."""
import math
from fractions import Fraction

import numpy as np


# ---- patch rows ---------------------------------------------------------------------------------------


def patch_size(width, height, patch, merge, min_pixels=0, max_pixels=0):
    """(height, width) in pixels that an image is resized to, by exact comparison of multiples."""
    u = patch * merge

    def nearest(side):
        return max(1, math.floor(Fraction(side, u) + Fraction(1, 2)))

    kh, kw = nearest(height), nearest(width)
    if max_pixels and kh * kw * u * u > max_pixels:
        # k u <= side sqrt(most / (w h))  <=>  k k u u w h <= side side most
        def down(side):
            k = 0
            while (k + 1) ** 2 * u * u * width * height <= side * side * max_pixels:
                k += 1
            return max(1, k)
        kh, kw = down(height), down(width)
    elif kh * kw * u * u < min_pixels:
        def up(side):
            k = 1
            while k * k * u * u * width * height < side * side * min_pixels:
                k += 1
            return k
        kh, kw = up(height), up(width)
    return kh * u, kw * u


def axis_weights(size, out, antialias):
    """[out, size] weights of one axis."""
    m = np.zeros((out, size))
    for i in range(out):
        centre = Fraction((2 * i + 1) * size, 2 * out) - Fraction(1, 2)
        support = max(Fraction(size, out), Fraction(1))
        if antialias and support > 1:
            for j in range(max(0, math.ceil(centre - support)), min(size - 1, math.floor(centre + support)) + 1):
                m[i, j] = float(1 - abs(j - centre) / support)
            m[i] /= m[i].sum()
        else:
            low = math.floor(centre)
            part = float(centre - low)
            m[i, min(max(low, 0), size - 1)] += 1 - part
            m[i, min(max(low + 1, 0), size - 1)] += part
    return m


def patch_rows(frames, out_h, out_w, patch, merge, group, antialias, mean, std):
    """frames uint8 [f, h, w, 3] -> float64 [rows, 3 * group * patch * patch]."""
    f, h, w, _ = frames.shape
    wy, wx = axis_weights(h, out_h, antialias), axis_weights(w, out_w, antialias)
    v = np.stack([np.stack([wy @ frame[..., c].astype(np.float64) @ wx.T for c in range(3)], -1) for frame in frames])
    v = (v / 255.0 - np.asarray(mean, dtype=np.float64)) / np.asarray(std, dtype=np.float64)
    rows = []
    for t in range(-(-f // group)):
        some = [v[min(t * group + k, f - 1)] for k in range(group)]
        for y0 in range(0, out_h, patch * merge):
            for x0 in range(0, out_w, patch * merge):
                for a in range(merge):
                    for b in range(merge):
                        y, x = y0 + a * patch, x0 + b * patch
                        rows.append(np.stack([[s[y:y + patch, x:x + patch, c] for s in some] for c in range(3)]).ravel())
    return np.stack(rows)


# ---- places -----------------------------------------------------------------------------------------------


def segment_valid(s):
    t, h, w, step = s
    if h == 0 and w == 0:
        return t >= 0 and step == 0
    return 0 <= t <= 32767 and 1 <= h <= 32767 and 1 <= w <= 32767 and 0 <= step <= 32767


def token_positions(sequences, first, merge):
    """Lists of (t, h, w, step) -> places [3, tokens] (Python ints), first token of each sequence, next places."""
    out, starts, nexts = [], [0], []
    for segments, p in zip(sequences, first):
        for t, h, w, step in segments:
            if not segment_valid((t, h, w, step)) or t == 0:
                continue
            if h == 0:
                out += [(p + j,) * 3 for j in range(t)]
                p += t
                continue
            order = [(y, x) for Y in range(0, h, merge) for X in range(0, w, merge)
                     for y in range(Y, min(Y + merge, h)) for x in range(X, min(X + merge, w))]
            out += [(p + a * step, p + y, p + x) for a in range(t) for y, x in order]
            p += max((t - 1) * step, h - 1, w - 1) + 1
        starts.append(len(out))
        nexts.append(p)
    return np.array(out, dtype=np.int64).reshape(-1, 3).T, starts, nexts


# ---- rotary embedding -------------------------------------------------------------------------------------------


def pair_axes(sections, interleaved):
    if not interleaved:
        return [a for a in range(3) for _ in range(sections[a])]
    return [i % 3 if i % 3 and i < 3 * sections[i % 3] else 0 for i in range(sum(sections))]


def frequencies(sections, base, interleaved, per_axis):
    """Radians a place for every pair, in extended precision."""
    axes = pair_axes(sections, interleaved)
    base = np.longdouble(base)
    if not per_axis:
        return [base ** (-np.longdouble(i) / np.longdouble(len(axes))) for i in range(len(axes))]
    return [base ** (-np.longdouble(axes[:i].count(a)) / np.longdouble(sections[a])) for i, a in enumerate(axes)]


def rotary(x, positions, axes, freqs, adjacent, inverse):
    """x [tokens, heads, dim] float64, positions [3, tokens] -> rotated, float64 (angles in extended precision)."""
    out = np.array(x, dtype=np.float64)
    n = len(axes)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
        angle = positions[axes[i]].astype(np.longdouble) * np.longdouble(freqs[i])
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        if inverse:
            s = -s
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return out


# ---- slots --------------------------------------------------------------------------------------------------------


def block_slots(cached, fresh, block_size, n_blocks, stack, table, capacity):
    """stack: free blocks, top last; table [n, width].  -> slots, table, token_starts, lengths, status, blocks left."""
    table, width = table.copy(), table.shape[1]
    slots, starts, lengths, status = [], [0], [], []
    asked, left = 0, len(stack)
    for i, (c, f) in enumerate(zip(cached, fresh)):
        c, f = int(c), int(f)
        if c < 0 or f < 0:
            starts.append(starts[-1])
            lengths.append(0)
            status.append(-1)
            continue
        had, want = -(-c // block_size), -(-(c + f) // block_size)
        starts.append(starts[-1] + f)
        good = want <= width and starts[-1] <= capacity and c + f < 2 ** 31
        if good:
            asked += want - had
            good = want == had or asked <= len(stack)
        if not good:
            slots += [-1] * f
            lengths.append(c)
            status.append(-2)
            continue
        if want > had:
            table[i, had:want] = stack[len(stack) - asked:len(stack) - asked + want - had][::-1]
            left = len(stack) - asked
        for p in range(c, c + f):
            b = int(table[i, p // block_size])
            slots.append(b * block_size + p % block_size if 0 <= b < n_blocks else -1)
        lengths.append(c + f)
        status.append(0)
    slots = (slots + [-1] * capacity)[:capacity]
    return np.array(slots, dtype=np.int64), table, np.array(starts), np.array(lengths), np.array(status), left
