"""Checks of the operators for packed batches of tokens, shared by the GPU tests and by the CPU build of the kernels.

A backend has put(array) -> buffer, ptr(buffer), get(buffer) -> array and sync().  Buffers are numpy arrays
of raw elements; bfloat16 is kept as its bits (uint16)."""
import math

import numpy as np

import paper_2411_19114_amd.binding as prep
from oracle import tokens as oracle

MEAN, STD = tuple(float(np.float32(v)) for v in (0.485, 0.456, 0.406)), tuple(float(np.float32(v)) for v in (0.229, 0.224, 0.225))
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # of a rounding, relative
LEAST_STEP = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # and absolute, near zero
NUMPY = {"f32": np.float32, "f16": np.float16, "bf16": np.uint16}
ULP = 2.0 ** -24


def pack(x, dtype):
    if dtype != "bf16":
        return np.asarray(x).astype(NUMPY[dtype])
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def unpack(x, dtype):
    return (x.astype(np.uint32) << 16).view(np.float32).astype(np.float64) if dtype == "bf16" else x.astype(np.float64)


def within(got, want, tolerance, dtype):
    """|got - want| up to `tolerance` plus the rounding to dtype."""
    limit = tolerance * (1 + HALF_STEP[dtype]) + np.abs(want) * HALF_STEP[dtype] + LEAST_STEP[dtype]
    over = np.abs(got - want) - limit
    assert np.isfinite(got).all()
    assert over.max(initial=-1.0) <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))


# ---- patch rows -------------------------------------------------------------------------------------------

# sizes (w, h) of the clips, frames, patch, merge, frames a patch, dtype, antialiased, min_pixels, max_pixels
PATCHES = {
    "one_pixel": ([(1, 1)], [1], 1, 1, 1, "f32", True, 0, 0),
    "one_pixel_enlarged": ([(1, 1)], [1], 5, 2, 2, "bf16", True, 0, 0),
    "narrow": ([(2, 60), (60, 2), (1, 33), (3, 3)], [1] * 4, 4, 2, 1, "f32", True, 0, 0),
    "odd": ([(37, 53), (64, 48)], [1, 1], 8, 2, 1, "bf16", True, 0, 0),
    "odd_two_taps": ([(37, 53), (64, 48)], [1, 1], 8, 2, 1, "f16", False, 0, 0),
    "reduced": ([(90, 71), (33, 120)], [1, 1], 7, 2, 2, "f16", True, 0, 28 * 42),
    "reduced_far": ([(150, 110)], [1], 4, 1, 1, "f32", True, 0, 200),
    "reduced_two_taps": ([(90, 71)], [1], 6, 1, 1, "f32", False, 0, 700),
    "enlarged": ([(20, 13)], [1], 4, 2, 1, "f32", True, 60 * 60, 0),
    "one_axis_each_way": ([(200, 9)], [1], 14, 1, 1, "f32", True, 0, 0),
    "clip": ([(30, 22), (17, 40)], [3, 4], 6, 1, 2, "bf16", True, 0, 400),
    "clip_longer_groups": ([(16, 16)], [5], 4, 2, 4, "f16", False, 0, 0),
    "patch_of_one": ([(9, 7)], [1], 1, 3, 1, "f32", True, 0, 0),
    "large_patch": ([(70, 60)], [1], 64, 1, 1, "bf16", True, 0, 0),
    "more_than_a_launch": ([(4 + i % 5, 4 + i % 3) for i in range(35)], [1] * 35, 4, 1, 1, "f16", True, 0, 0),
    "several_tiles": ([(203, 90), (90, 203)], [1, 2], 14, 2, 2, "bf16", True, 0, 0),
    "several_tiles_reduced": ([(310, 190)], [1], 7, 3, 1, "f16", True, 0, 120 * 120),
    "several_tiles_two_taps": ([(150, 131)], [1], 16, 1, 1, "f32", False, 0, 100 * 100),
    "tall_patches": ([(150, 200)], [1], 50, 1, 2, "f16", True, 0, 0),
    "reduced_beyond_tiles": ([(400, 60), (40, 400)], [1, 1], 2, 1, 1, "f32", True, 0, 40),
    "few_columns": ([(7, 40), (6, 50), (5, 33), (8, 20)], [1] * 4, 4, 1, 1, "f16", True, 0, 0),
    "wide_window": ([(50, 46)], [1], 3, 5, 1, "f32", True, 0, 0),
}


# more tiles than a GPU holds at a time, so that workgroups take several
PATCHES_LARGE = {
    "large_photos": ([(640, 480), (333, 517), (500, 375)] * 4, [1] * 12, 14, 2, 2, "bf16", True, 0, 0),
    "large_clip": ([(900, 700)], [7], 14, 2, 2, "f16", True, 0, 400 * 300),
    "large_parts": ([(900, 700)], [3], 40, 1, 1, "bf16", True, 0, 0),
    "large_two_taps": ([(640, 480)] * 70, [1] * 70, 16, 1, 1, "f32", False, 0, 300 * 300),
    "large_strong": ([(1500, 1200)], [2], 7, 2, 1, "f32", True, 0, 250 * 200),
}


def picture(rng, shape):
    """Noise, flat stretches and the extremes."""
    v = rng.integers(0, 256, shape)
    v[rng.random(shape) < 0.1] = 255
    v[rng.random(shape) < 0.1] = 0
    if v.shape[1] > 4:
        v[:, :v.shape[1] // 4] = 200
    return v.astype(np.uint8)


def patch_tolerance(w, h, out_w, out_h, antialias):
    """Of a normalized value before its last rounding.  Per axis with half-width s and at most 2 s + 1 taps: a weight is
    1 - |j - c| / s from values rounded three times, so off by at most 4 steps of 2^-24, the weights' sum is at least s / 2 (the triangle's
    half at a border), so the mean moves by at most 255 (2 s + 1) 4 / (s / 2) <= 255 * 24 steps; adding up the taps rounds 2 s + 1
    times, weights' sum and division 2 s + 3 more.  Then the scale, the offset and their sum."""
    steps = 0.0
    for size, out in ((w, out_w), (h, out_h)):
        s = max(1.0, size / out) if antialias else 1.0
        steps += 24 + 2 * s + 1 + 2 * s + 3
    scale = max(1 / s for s in STD)
    return (steps * scale + 3 * (scale + max(m / s for m, s in zip(MEAN, STD)))) * ULP


def check_patches(backend, name, seed=0, out_pad=3, pitch_pad=4, lead=5):
    sizes, frames, patch, merge, group, dtype, antialias, least, most = (PATCHES | PATCHES_LARGE)[name]
    rng = np.random.default_rng(seed)
    params = prep.make_patch_params(patch, merge, group, dtype, MEAN, STD, prep.FILTER_ANTIALIAS if antialias else prep.FILTER_BILINEAR,
                                    min_pixels=least, max_pixels=most)
    clips, offsets, pitches, strides, want, at, starts = [], [], [], [], [], lead, [0]
    for i, ((w, h), f) in enumerate(zip(sizes, frames)):
        clip = picture(rng, (f, h, w, 3))
        oh, ow = oracle.patch_size(w, h, patch, merge, least, most)
        grid = prep.patch_grid(params, w, h, f)
        assert grid == (-(-f // group), oh // patch, ow // patch)
        pitch = 3 * w + (pitch_pad if i % 2 else 0)
        stride = pitch * h + (7 if i % 2 else 0)
        clips.append(clip)
        offsets.append(at)
        pitches.append(pitch)
        strides.append(stride)
        at += stride * f
        want.append((oracle.patch_rows(clip, oh, ow, patch, merge, group, antialias, MEAN, STD), patch_tolerance(w, h, ow, oh, antialias)))
        starts.append(starts[-1] + math.prod(grid))
    # the last clip ends with its last pixel
    last = offsets[-1] + strides[-1] * (frames[-1] - 1) + pitches[-1] * (sizes[-1][1] - 1) + 3 * sizes[-1][0]
    rgb = np.full(max(at, last), 77, dtype=np.uint8)
    for clip, offset, pitch, stride in zip(clips, offsets, pitches, strides):
        f, h, w, _ = clip.shape
        for k in range(f):
            for y in range(h):
                rgb[offset + k * stride + y * pitch:][:3 * w] = clip[k, y].ravel()
    row = 3 * group * patch * patch
    filler = pack(np.full((starts[-1] + 2, row + out_pad), -77.0), dtype)
    out, src = backend.put(filler), backend.put(rgb[:last])
    still = all(f == 1 for f in frames) and seed % 2 == 0
    got_starts = prep.patch_rows(0, backend.ptr(src), offsets, [s[0] for s in sizes], [s[1] for s in sizes], pitches, params, backend.ptr(out),
                                 starts[-1], frames=None if still else frames, frame_strides=None if still else strides,
                                 out_stride=row + out_pad, stream=backend.stream)
    assert got_starts == starts
    got = backend.get(out)
    assert (got[:, row:] == filler[:, row:]).all() and (got[starts[-1]:] == filler[starts[-1]:]).all()
    for i, (rows, tolerance) in enumerate(want):
        within(unpack(got[starts[i]:starts[i + 1], :row], dtype), rows, tolerance, dtype)


# ---- places -------------------------------------------------------------------------------------------------

T, G = lambda n: (n, 0, 0, 0), lambda t, h, w, step=1: (t, h, w, step)
# sequences of segments, merge, room behind (negative: too little), places of the first tokens
POSITIONS = {
    "none": ([], 1, 5, None),
    "empty_sequences": ([[], [T(0)], [], [T(3)], []], 1, 4, [5, 6, 7, 8, 9]),
    "one_token": ([[T(1)]], 1, 0, [41]),
    "text": ([[T(3), T(4)], [T(300)]], 1, 3, None),
    "picture": ([[T(2), G(1, 3, 5), T(2)], [G(1, 7, 2)]], 1, 0, None),
    "clip": ([[G(4, 2, 3, 5), T(1)], [T(1), G(3, 1, 1, 0), T(2)], [G(0, 4, 4), T(1)]], 1, 2, [0, 100, 7]),
    "merged": ([[G(2, 4, 6), G(1, 2, 2)], [T(3), G(1, 8, 4)]], 2, 1, None),
    "merged_ragged": ([[G(1, 7, 5), T(2), G(3, 1, 7, 2), G(2, 8, 1)]], 3, 0, [9]),
    "refused_segments": ([[T(2), (-3, 0, 0, 0), (2, 3, 0, 1), (2, 0, 3, 1), (1, -1, 4, 1), (40000, 1, 1, 1), (1, 1, 1, -1), (3, 0, 0, 2), T(2)],
                          [(2, 32768, 1, 1), T(1)]], 1, 3, None),
    "too_little_room": ([[T(5), G(2, 3, 3)], [T(9)]], 2, -11, None),
    "no_room": ([[T(5)], [T(2)]], 1, -7, None),
    "wraps": ([[T(6)], [T(2)]], 1, 0, [2 ** 31 - 3, -4]),
    "long_steps": ([[G(3, 1, 2, 32767), T(1)]], 1, 0, None),
    "long_list": ([[T(i % 2), G(1, 1, 1 + i % 2)] * 50 for i in range(45)], 1, 2, list(range(45))),
    "many_sequences": ([[T(i % 3)] if i % 5 else [] for i in range(4300)], 1, 0, None),
    "many_segments": ([[T(1 + i % 3), G(1, 1 + i % 2, 2)] * 40 for i in range(30)], 2, 9, list(range(30))),
}


def check_positions(backend, name, workspace_pad=0, misaligned=0):
    sequences, merge, room, first = POSITIONS[name]
    n = len(sequences)
    want, starts, nexts = oracle.token_positions(sequences, first or [0] * n, merge)
    capacity = starts[-1] + room
    flat = [s for q in sequences for s in q]
    bounds = np.cumsum([0] + [len(q) for q in sequences]).astype(np.int32)
    segments = backend.put(np.array(flat, dtype=np.int32).reshape(-1, 4))
    seq, base = backend.put(bounds), backend.put(np.array(first, dtype=np.int32)) if first else None
    positions = backend.put(np.full(3 * capacity + 1 + misaligned, 77, dtype=np.int32))
    token_starts, nxt = backend.put(np.full(n + 2, 77, dtype=np.int32)), backend.put(np.full(n + 1, 77, dtype=np.int32))
    size = prep.token_positions_workspace(len(flat)) + workspace_pad
    work = backend.put(np.full(size, 77, dtype=np.uint8))
    prep.token_positions(backend.ptr(segments), len(flat), backend.ptr(seq), n, backend.ptr(base) if first else 0, merge,
                         backend.ptr(positions) + 4 * misaligned, capacity, backend.ptr(token_starts), backend.ptr(nxt), backend.ptr(work), size,
                         stream=backend.stream)
    full = np.zeros((3, capacity), dtype=np.int64)
    full[:, :starts[-1]] = want[:, :capacity]
    got = backend.get(positions)
    assert (got[:misaligned] == 77).all() and got[-1] == 77
    assert np.array_equal(got[misaligned:-1].reshape(3, capacity), full.astype(np.uint32).astype(np.int32))
    assert backend.get(token_starts).tolist() == starts + [77]
    assert backend.get(nxt).tolist() == np.array(nexts, dtype=np.int64).astype(np.uint32).astype(np.int32).tolist() + [77]


# ---- slots ------------------------------------------------------------------------------------------------------

# cached, fresh, block size, table width, blocks left on the stack beyond those needed, room for tokens beyond those there
SLOTS = {
    "none": ([], [], 16, 4, 3, 5),
    "one_token": ([0], [1], 16, 1, 0, 0),
    "step": ([5, 16, 31, 0, 32], [1] * 5, 16, 4, 2, 3),
    "nothing_new": ([5, 0, 16], [0, 0, 0], 16, 4, 1, 2),
    "prompts": ([0, 7, 40], [50, 9, 100], 8, 20, 5, 0),
    "block_of_one": ([0, 3], [4, 2], 1, 8, 0, 1),
    "large_blocks": ([100, 0], [300, 1000], 256, 5, 1, 0),
    "odd_blocks": ([10, 0, 21], [30, 8, 7], 7, 6, 0, 2),
    "too_few_blocks": ([0, 8, 0, 3, 8], [16, 9, 8, 2, 8], 8, 4, -2, 0),
    "no_blocks": ([0, 7], [4, 1], 8, 4, -1, 0),
    "short_table": ([0, 0, 8], [33, 16, 8], 8, 4, 3, 0),
    "too_little_room": ([0, 0, 0], [5, 6, 7], 4, 4, 2, -4),
    "no_room": ([3], [4], 4, 4, 2, -4),
    "negative": ([0, -1, 4, 2 ** 31 - 1], [5, 3, -2, 2], 4, 4, 2, 1),
    "long_list": ([(i * 7) % 50 for i in range(4200)], [(i * 5) % 3 for i in range(4200)], 4, 16, -3, 5),
    "many": ([(i * 7) % 50 for i in range(1500)], [(i * 5) % 4 for i in range(1500)], 4, 16, 7, 11),
}


def check_slots(backend, name, table_pad=2, bad_ids=False):
    cached, fresh, block, width, spare, room = SLOTS[name]
    n = len(cached)
    rng = np.random.default_rng(3)
    ok = [c >= 0 and f >= 0 for c, f in zip(cached, fresh)]
    had = [min(-(-c // block), width) if o else 0 for c, o in zip(cached, ok)]
    need = [max(0, min(-(-(c + f) // block), width) - h) if o else 0 for c, f, o, h in zip(cached, fresh, ok, had)]
    n_blocks = sum(had) + sum(need) + abs(spare) + 3
    ids = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((n, width), 55, dtype=np.int32)
    for i in range(n):
        table[i, :had[i]] = ids[sum(had[:i]):sum(had[:i]) + had[i]]
    stack = ids[sum(had):sum(had) + max(0, sum(need) + spare)]
    if bad_ids and len(stack) > 1 and n > 0:
        stack[-1], stack[0] = n_blocks, -5
        table[0, 0] = -9 if had[0] else table[0, 0]
    capacity = sum(f for f, o in zip(fresh, ok) if o) + room
    want = oracle.block_slots(cached, fresh, block, n_blocks, stack, table, capacity)
    padded = np.full((n, width + table_pad), 55, dtype=np.int32)
    padded[:, :width] = table
    dev = {"cached": np.array(cached, dtype=np.int32), "fresh": np.array(fresh, dtype=np.int32), "free": np.concatenate([stack, [99, 99]]).astype(np.int32),
           "count": np.array([len(stack)], dtype=np.int32), "table": padded, "slots": np.full(capacity + 1, 77, dtype=np.int64),
           "starts": np.full(n + 2, 77, dtype=np.int32), "lengths": np.full(n + 1, 77, dtype=np.int32), "status": np.full(n + 1, 77, dtype=np.int32),
           "left": np.full(2, 77, dtype=np.int32), "work": np.full(prep.block_slots_workspace(n), 77, dtype=np.uint8)}
    before = {k: v.copy() for k, v in dev.items()}
    dev = {k: backend.put(v) for k, v in dev.items()}
    p = {k: backend.ptr(v) for k, v in dev.items()}
    prep.block_slots(n, block, n_blocks, p["cached"], p["fresh"], p["free"], len(stack), p["count"], p["table"], width + table_pad, width,
                     p["slots"], capacity, p["starts"], p["lengths"], p["status"], p["left"], p["work"], len(before["work"]), stream=backend.stream)
    got = {k: backend.get(v) for k, v in dev.items()}
    for k in ("cached", "fresh", "free", "count"):
        assert np.array_equal(got[k], before[k]), k
    assert np.array_equal(got["slots"], np.append(want[0], 77))
    assert np.array_equal(got["table"][:, :width], want[1]) and (got["table"][:, width:] == 55).all()
    assert np.array_equal(got["starts"], np.append(want[2], 77))
    assert np.array_equal(got["lengths"], np.append(want[3], 77))
    assert np.array_equal(got["status"], np.append(want[4], 77))
    assert got["left"].tolist() == [want[5], 77]


# ---- rotary embedding ----------------------------------------------------------------------------------------------

# tokens, q heads, k heads, dim, sections, dtype, adjacent, interleaved, per axis, base, farthest place, layout, what
ROTARY = {
    "least": (1, 1, 0, 2, (1, 0, 0), "f32", False, False, False, 1e4, 10, "plain", ""),
    "one_token": (1, 4, 2, 64, (32, 0, 0), "bf16", False, False, False, 1e4, 100000, "plain", ""),
    "text": (37, 3, 1, 64, (32, 0, 0), "bf16", False, False, False, 5e5, 100000, "plain", ""),
    "sections": (19, 4, 2, 128, (16, 24, 24), "bf16", False, False, False, 1e6, 30000, "fused", ""),
    "sections_f16": (19, 4, 2, 128, (16, 24, 24), "f16", False, False, False, 1e6, 30000, "plain", ""),
    "interleaved": (9, 2, 2, 32, (8, 4, 4), "f32", False, True, False, 1e4, 500, "plain", ""),
    "adjacent": (13, 2, 1, 64, (12, 10, 10), "f32", True, True, False, 1e4, 5000, "plain", ""),
    "adjacent_bf16": (21, 5, 1, 96, (48, 0, 0), "bf16", True, False, False, 1e4, 5000, "fused", ""),
    "encoder": (25, 4, 4, 80, (0, 20, 20), "f16", False, False, True, 1e4, 140, "fused", ""),
    "partial": (11, 2, 1, 96, (16, 4, 4), "bf16", False, False, False, 1e4, 4000, "plain", ""),
    "partial_adjacent": (11, 2, 1, 40, (3, 1, 1), "f16", True, False, False, 1e4, 4000, "plain", ""),
    "odd_dim": (7, 2, 1, 33, (10, 3, 2), "f32", False, False, False, 1e4, 900, "plain", ""),
    "odd_pairs": (7, 2, 1, 30, (5, 5, 5), "bf16", False, True, False, 1e4, 900, "plain", ""),
    "wide": (3, 1, 1, 1024, (512, 0, 0), "f16", False, False, False, 1e4, 900, "plain", ""),
    "far": (16, 1, 1, 128, (22, 21, 21), "f32", False, True, False, 1e6, 2 ** 31 - 1, "plain", ""),
    "far_back": (16, 1, 1, 16, (3, 3, 2), "f32", False, False, False, 1e4, -2 ** 31, "plain", ""),
    "head_major": (10, 3, 2, 64, (12, 10, 10), "bf16", False, False, False, 1e4, 400, "head_major", ""),
    "shared_input": (6, 4, 4, 64, (32, 0, 0), "f16", False, False, False, 1e4, 400, "shared", ""),
    "unaligned": (9, 2, 1, 64, (32, 0, 0), "bf16", False, False, False, 1e4, 400, "shifted", ""),
    "in_place": (17, 3, 2, 64, (32, 0, 0), "bf16", False, False, False, 1e4, 400, "fused", "in_place"),
    "in_place_adjacent": (17, 3, 2, 20, (6, 2, 2), "f32", True, False, False, 1e4, 400, "plain", "in_place"),
    "back": (14, 3, 2, 64, (12, 10, 10), "f32", False, False, False, 1e4, 400, "plain", "inverse"),
    "back_adjacent": (14, 3, 2, 48, (12, 6, 6), "bf16", True, True, False, 1e4, 400, "fused", "inverse"),
    "only_keys": (5, 0, 3, 64, (32, 0, 0), "bf16", False, False, False, 1e4, 400, "plain", ""),
    "store": (23, 4, 2, 64, (12, 10, 10), "bf16", False, False, False, 1e4, 400, "fused", "store"),
    "store_f32": (23, 2, 1, 36, (8, 4, 4), "f32", False, False, False, 1e4, 400, "plain", "store"),
    "store_and_out": (12, 2, 2, 128, (64, 0, 0), "f16", False, False, False, 1e4, 400, "plain", "store keep"),
    "store_head_major": (18, 2, 3, 32, (6, 5, 5), "bf16", True, False, False, 1e4, 400, "plain", "store major"),
    "store_partial": (9, 1, 1, 80, (12, 0, 0), "bf16", False, False, False, 1e4, 400, "fused", "store"),
    "store_one": (1, 8, 1, 128, (64, 0, 0), "bf16", False, False, False, 1e4, 400, "fused", "store"),
    "store_only_keys": (6, 0, 2, 64, (32, 0, 0), "f16", False, False, False, 1e4, 400, "fused", "store"),
    "one_head": (300, 1, 0, 32, (16, 0, 0), "bf16", False, False, False, 1e4, 400, "plain", ""),
    "many_heads": (5, 33, 7, 24, (12, 0, 0), "bf16", False, False, False, 1e4, 400, "plain", ""),
}
# calls of many rows (a GPU's)
ROTARY_LARGE = {
    "large_one_head": (40000, 1, 1, 32, (16, 0, 0), "bf16", False, False, False, 1e4, 400, "plain", ""),
    "large_lines": (2100, 14, 2, 128, (16, 24, 24), "bf16", False, False, False, 1e6, 30000, "fused", "store"),
    "large_lines_f32": (3000, 9, 3, 64, (12, 10, 10), "f32", True, True, False, 1e4, 5000, "plain", "inverse"),
    "large_pieces": (3001, 8, 8, 80, (0, 20, 20), "f16", False, False, True, 1e4, 140, "fused", ""),
    "large_in_place": (2500, 14, 2, 128, (64, 0, 0), "f16", False, False, False, 1e4, 9000, "fused", "in_place"),
    "large_pairs": (700, 5, 2, 50, (9, 8, 8), "bf16", True, False, False, 1e4, 9000, "plain", ""),
}
# |error of cos or sin|: the angle is an eighth of a turn at most, rounded twice (as a float, times 2 pi / 2^32) and cut at 2^-33 of a
# turn; the series' remainder; its evaluation, two roundings of values up to 1 that count in full (the others are scaled by x^2 / 2 < 0.31)
TRIG = (math.pi / 4) * 2 * ULP + 2 * math.pi * 2.0 ** -33 + 2e-9 + 3 * ULP


def rotary_tolerance(x, n, adjacent):
    """Of a rotated value before its last rounding: both terms' cos or sin, the smaller product's rounding, the sum's."""
    out = np.zeros(x.shape)
    m = np.abs(x[..., 0:2 * n:2]) + np.abs(x[..., 1:2 * n:2]) if adjacent else np.abs(x[..., :n]) + np.abs(x[..., n:2 * n])
    m = m * (TRIG + 2 * ULP)
    if adjacent:
        out[..., 0:2 * n:2] = out[..., 1:2 * n:2] = m
    else:
        out[..., :n] = out[..., n:2 * n] = m
    return out


class Laid:
    """[tokens, heads, dim] values laid out in a buffer."""

    def __init__(self, backend, values, dtype, layout, shift=0):
        n, h, d = values.shape
        if layout == "head_major":
            self.strides, size = (d, n * d), n * h * d
        elif layout == "shared":
            self.strides, size = (d, 0), n * d
        elif layout == "gaps":
            self.strides, size = (h * (d + 8) + 16, d + 8), n * (h * (d + 8) + 16)
        else:
            self.strides, size = (h * d, d), n * h * d
        self.backend, self.dtype, self.shape, self.shift = backend, dtype, values.shape, shift
        raw = pack(np.full(size + shift + 3, 77.0), dtype)
        self.index = shift + np.arange(n)[:, None, None] * self.strides[0] + np.arange(h)[None, :, None] * self.strides[1] + np.arange(d)
        raw[self.index] = pack(values, dtype)
        self.before = raw.copy()
        self.buffer = backend.put(raw)

    def view(self):
        return self.backend.ptr(self.buffer) + self.shift * self.before.itemsize, self.strides[0], self.strides[1]

    def values(self):
        got = self.backend.get(self.buffer)
        rest = np.ones(len(got), dtype=bool)
        rest[self.index.ravel()] = False
        assert np.array_equal(got[rest], self.before[rest]), "written outside its rows"
        return unpack(got[self.index], self.dtype)


def check_rotary(backend, name, seed=0):
    n, qh, kh, d, sections, dtype, adjacent, interleaved, per_axis, base, reach, layout, what = (ROTARY | ROTARY_LARGE)[name]
    rng = np.random.default_rng(seed + 11)
    inverse, store = "inverse" in what, "store" in what
    low, high = sorted((0, reach))
    positions = rng.integers(low, high, (3, n + 2), endpoint=True)
    positions[:, :1] = reach  # the farthest place itself
    pairs = sum(sections)
    axes, freqs = oracle.pair_axes(sections, interleaved), oracle.frequencies(sections, base, interleaved, per_axis)

    def values(heads):
        x = rng.standard_normal((n, max(heads, 1), d)) * np.exp(rng.uniform(-3, 3, (n, max(heads, 1), 1)))
        if layout == "shared":
            x[:] = x[:, :1]
        return unpack(pack(x, dtype), dtype)

    q, k, v = values(qh), values(kh), values(kh)
    shift = 1 if layout == "shifted" else 0
    if layout == "fused":  # one projection's output
        whole = Laid(backend, np.concatenate([q, k, v], 1), dtype, "plain")
        heads = whole.shape[1]
        p, size = backend.ptr(whole.buffer), whole.before.itemsize
        views = [(p + at * d * size, heads * d, d) for at in (0, q.shape[1], q.shape[1] + k.shape[1])]
    else:
        laid = [Laid(backend, x, dtype, layout, shift) for x in (q, k, v)]
        views = [x.view() for x in laid]
    args = dict(q_heads=qh, k_heads=kh, inverse=inverse)
    filler = np.full
    out_layout = "gaps" if layout in ("plain", "shared") else "head_major" if layout == "head_major" else "plain"
    q_out = Laid(backend, filler(q.shape, 55.0), dtype, out_layout, shift)
    k_out = Laid(backend, filler(k.shape, 55.0), dtype, out_layout, shift)
    if qh:
        args.update(q=views[0], q_out=views[0] if what == "in_place" else q_out.view())
    if kh:
        args.update(k=views[1])
        if not store or "keep" in what:
            args.update(k_out=views[1] if what == "in_place" else k_out.view())
    if store:
        block, n_blocks = 4, n // 4 + 3
        order = (0, 2, 1, 3) if "major" in what else (0, 1, 2, 3)  # heads before the places of a block
        shape = [(n_blocks, block, kh, d)[a] for a in order]
        caches = [pack(rng.standard_normal(shape), dtype) for _ in range(2)]
        buffers = [backend.put(c) for c in caches]
        slots = rng.permutation(n_blocks * block)[:n].astype(np.int64)
        slots[rng.random(n) < 0.2] = -1
        if n > 4:
            slots[1], slots[3] = n_blocks * block, 2 ** 40
        on_device = backend.put(slots)
        strides = np.array(caches[0].strides)[np.argsort(order)] // caches[0].itemsize
        args.update(v=views[2], k_cache=backend.ptr(buffers[0]), v_cache=backend.ptr(buffers[1]), n_blocks=n_blocks, block_size=block,
                    block_stride=int(strides[0]), slot_stride=int(strides[1]), cache_head_stride=int(strides[2]), slots=backend.ptr(on_device))
    places = backend.put(positions.astype(np.int32))
    rotary = prep.Rotary(d, sections, base, dtype, pairing=int(adjacent), order=int(interleaved), per_axis=per_axis)
    rotary.apply(n, backend.ptr(places), n + 2, stream=backend.stream, **args)
    backend.sync()
    rotary.close()
    places = positions[:, :n]
    want_q, want_k = (oracle.rotary(x, places, axes, freqs, adjacent, inverse) for x in (q, k))
    if what == "in_place":
        if layout == "fused":
            got = whole.values()
            got_q, got_k, rest = got[:, :qh], got[:, qh:qh + kh], got[:, qh + kh:]
            assert np.array_equal(rest, v)
        else:
            got_q, got_k = laid[0].values(), laid[1].values()
    else:
        got_q, got_k = q_out.values(), k_out.values()
        for x, before in ([(whole, np.concatenate([q, k, v], 1))] if layout == "fused" else zip(laid, (q, k, v))):
            assert np.array_equal(x.values(), before), "an input was written"
    if qh:
        within(got_q, want_q, rotary_tolerance(q, pairs, adjacent), dtype)
        assert np.array_equal(got_q[..., 2 * pairs:], q[..., 2 * pairs:])
    if kh and "k_out" in args:
        within(got_k, want_k, rotary_tolerance(k, pairs, adjacent), dtype)
    if store:
        stored = np.flatnonzero((slots >= 0) & (slots < n_blocks * block))
        kept = np.ones(n_blocks * block, dtype=bool)
        kept[slots[stored]] = False
        for buffer, cache, want, x in zip(buffers, caches, (want_k, v), (k, None)):
            got = backend.get(buffer).transpose(np.argsort(order)).reshape(n_blocks * block, kh, d)
            assert np.array_equal(got[kept], cache.transpose(np.argsort(order)).reshape(n_blocks * block, kh, d)[kept])
            got = unpack(got[slots[stored]], dtype)
            if x is None:
                assert np.array_equal(got, v[stored])
            else:
                within(got, want[stored], rotary_tolerance(k, pairs, adjacent)[stored], dtype)


def check_rotary_gradient(backend, adjacent):
    """The inverse is the gradient: against differences of the forward pass (which is linear, so that a wide step is exact up to rounding)."""
    n, h, d, sections = 6, 2, 24, (5, 3, 2)
    rng = np.random.default_rng(5)
    positions = backend.put(rng.integers(0, 3000, (3, n)).astype(np.int32))
    rotary = prep.Rotary(d, sections, 1e4, "f32", pairing=int(adjacent))

    def run(x, inverse):
        a, b = (backend.put(v.astype(np.float32)) for v in (x, np.zeros_like(x)))
        view = [(backend.ptr(v), h * d, d) for v in (a, b)]
        rotary.apply(n, backend.ptr(positions), n, q=view[0], q_out=view[1], q_heads=h, inverse=inverse, stream=backend.stream)
        return backend.get(b).astype(np.float64)

    x, g = (rng.standard_normal((n, h, d)).astype(np.float32).astype(np.float64) for _ in range(2))
    grad = run(g, True)
    step = 1.0
    for i in range(d):
        e = np.zeros_like(x)
        e[..., i] = step
        # (x + e is rounded to fp32: by at most half a step of 2^-24 * 8)
        slope = ((run(x + e, False) - run(x - e, False)) * g).sum(-1) / (2 * step)
        # every value of the two passes is off by (TRIG + 2 ULP) (|a| + |b|) + ULP |out| and its input by 4 ULP; two values of a head differ
        bound = (np.abs(g).max() * 2 * 2 * (np.abs(x).max() + step) * (2 * (TRIG + 2 * ULP) + ULP + 8 * ULP)) / (2 * step) * d / 2 + 4 * ULP * np.abs(g).max()
        assert np.abs(slope - grad[..., i]).max() <= bound
    # and there and back is where it began: an orthogonal map and its transpose, each off as above
    back = run(run(x, False), True)
    assert np.abs(back - x).max() <= 2 * np.abs(x).max() * 2 * (TRIG + 4 * ULP) * 1.5
    rotary.close()


# ---- refusals ---------------------------------------------------------------------------------------------------------


def refused(code, call, *args, **kwargs):
    try:
        call(*args, **kwargs)
    except prep.PrepError as e:
        assert e.code == code, (e.code, code)
        return
    raise AssertionError("not refused")


def check_patch_refusals(backend):
    src, out = backend.put(np.zeros(3000, dtype=np.uint8)), backend.put(np.full(4000, 7.0, dtype=np.float32))
    p, o = backend.ptr(src), backend.ptr(out)
    good = dict(patch=4, merge=2, frames_per_patch=1, out_dtype="f32", mean=MEAN, std=STD)
    make = lambda **kw: prep.make_patch_params(**{**good, **kw})  # noqa: E731
    E, L = prep.E_INVALID_ARG, prep.E_TOO_LARGE

    def call(code, params=None, offsets=(0,), w=(16,), h=(8,), pitch=(48,), out_ptr=None, rows=100, src_ptr=p, **kw):
        refused(code, prep.patch_rows, 0, src_ptr, list(offsets), list(w), list(h), list(pitch), params or make(), o if out_ptr is None else out_ptr, rows,
                stream=backend.stream, **kw)

    for kw in (dict(patch=0), dict(patch=65), dict(merge=0), dict(merge=17), dict(frames_per_patch=0), dict(frames_per_patch=17),
               dict(out_dtype=prep.U8_NHWC), dict(out_dtype=7), dict(filter=2), dict(min_pixels=-1), dict(max_pixels=-1), dict(std=(0, 1, 1)),
               dict(std=(1, float("nan"), 1)), dict(std=(1, float("inf"), 1)), dict(mean=(0, 0, float("inf"))), dict(min_pixels=1 << 40)):
        call(E, make(**kw))
    call(E, w=(0,))
    call(E, h=(0,))
    call(E, w=(65536,), pitch=(3 * 65536,))
    call(E, pitch=(47,))
    call(E, frames=[0], frame_strides=[400])
    call(E, frames=[2], frame_strides=[48 * 7 + 47])
    call(E, out_stride=47)
    call(E, out_ptr=o + 2)
    call(E, out_ptr=0)
    call(E, src_ptr=0)
    call(E, rows=-1)
    call(L, rows=7)  # 2 x 4 patches
    call(E, make(min_pixels=60000 * 60000), w=(65535,), h=(1,), pitch=(3 * 65535,))
    refused(E, prep.patch_grid, make(), 16, 8, 0)
    refused(E, prep.patch_grid, make(patch=64, merge=16), 65535, 65535)
    backend.sync()
    assert (backend.get(out) == 7.0).all()
    # no clips are none
    assert prep.patch_rows(0, p, [], [], [], [], make(), o, 0, stream=backend.stream) == [0]


def check_packing_refusals(backend):
    ints = backend.put(np.zeros(4096, dtype=np.int64))
    p = backend.ptr(ints)
    E, L = prep.E_INVALID_ARG, prep.E_TOO_LARGE
    good = dict(segments_ptr=p, n_segments=2, seq_segments_ptr=p, n_seq=1, first_ptr=0, merge=1, positions_ptr=p + 4096, capacity=8,
                token_starts_ptr=p + 8192, next_ptr=0, workspace_ptr=p + 16384, workspace_bytes=1024, stream=backend.stream)
    for kw in (dict(n_segments=-1), dict(n_segments=(1 << 20) + 1), dict(n_seq=-1), dict(n_seq=65536), dict(merge=0), dict(merge=32768),
               dict(capacity=-1), dict(capacity=2 ** 31), dict(segments_ptr=0), dict(seq_segments_ptr=0), dict(positions_ptr=0),
               dict(token_starts_ptr=0), dict(workspace_ptr=0), dict(segments_ptr=p + 2), dict(positions_ptr=p + 1), dict(first_ptr=p + 3),
               dict(next_ptr=p + 2), dict(first_ptr=p + 64, next_ptr=p + 64), dict(token_starts_ptr=p), dict(workspace_ptr=p + 8), dict(token_starts_ptr=p + 1), dict(seq_segments_ptr=p + 1)):
        refused(E, prep.token_positions, **{**good, **kw})
    refused(L, prep.token_positions, **{**good, "workspace_bytes": prep.token_positions_workspace(2) - 1})
    assert prep.token_positions_workspace(-1) == 0 and prep.token_positions_workspace((1 << 20) + 1) == 0
    good = dict(n=2, block_size=4, n_blocks=9, cached_ptr=p, fresh_ptr=p + 64, free_blocks_ptr=p + 128, free_capacity=4, free_count_ptr=p + 256,
                table_ptr=p + 512, table_stride=4, table_width=4, slots_ptr=p + 1024, capacity=8, token_starts_ptr=p + 2048,
                lengths_ptr=p + 2304, status_ptr=p + 2560, free_left_ptr=p + 2816, workspace_ptr=p + 4096, workspace_bytes=1024, stream=backend.stream)
    for kw in (dict(n=-1), dict(n=(1 << 20) + 1), dict(block_size=0), dict(block_size=65537), dict(n_blocks=-1), dict(n_blocks=2 ** 31),
               dict(free_capacity=-1), dict(table_width=-1), dict(table_stride=3), dict(capacity=-1), dict(capacity=2 ** 31), dict(cached_ptr=0),
               dict(fresh_ptr=0), dict(free_blocks_ptr=0), dict(free_count_ptr=0), dict(table_ptr=0), dict(slots_ptr=0), dict(token_starts_ptr=0),
               dict(lengths_ptr=0), dict(status_ptr=0), dict(free_left_ptr=0), dict(free_left_ptr=p + 256), dict(lengths_ptr=p), dict(status_ptr=p + 64), dict(workspace_ptr=0),
               dict(slots_ptr=p + 4), dict(cached_ptr=p + 1), dict(table_ptr=p + 2), dict(workspace_ptr=p + 4)):
        refused(E, prep.block_slots, **{**good, **kw})
    refused(L, prep.block_slots, **{**good, "workspace_bytes": prep.block_slots_workspace(2) - 1})
    assert prep.block_slots_workspace(-1) == 0 and prep.block_slots_workspace((1 << 20) + 1) == 0
    backend.sync()
    assert (backend.get(ints) == 0).all()


def check_rotary_refusals(backend):
    E = prep.E_INVALID_ARG
    good = dict(head_dim=16, sections=(8, 0, 0), base=1e4, dtype="f32")
    for kw in (dict(head_dim=1), dict(head_dim=1025), dict(sections=(9, 0, 0)), dict(sections=(0, 0, 0)), dict(sections=(9, -1, 0)),
               dict(dtype=prep.U8_NHWC), dict(pairing=2), dict(order=2), dict(base=0.0), dict(base=-1.0), dict(base=float("nan")),
               dict(sections=(0, 8, 0), order=1), dict(sections=(2, 0, 4), order=1), dict(frequencies=[float("inf")] * 8),
               dict(frequencies=[1.0] * 7)):
        refused(E, prep.Rotary, **{**good, **kw})
    refused(prep.E_HIP, prep.Rotary, **{**good, "device": 99})
    data = backend.put(np.zeros(8192, dtype=np.float32))
    p = backend.ptr(data)
    r = prep.Rotary(**good)
    n = 3
    good = dict(n_tokens=n, positions=p, axis_stride=n, q=(p + 1024, 32, 16), q_out=(p + 4096, 32, 16), q_heads=2, k=(p + 2048, 16, 16),
                k_out=(p + 8192, 16, 16), k_heads=1, stream=backend.stream)
    cache = dict(v=(p + 2560, 16, 16), k_cache=p + 12288, v_cache=p + 16384, n_blocks=2, block_size=2, block_stride=32, slot_stride=16,
                 cache_head_stride=16, slots=p + 20480)
    bad = [dict(n_tokens=-1), dict(n_tokens=2 ** 31), dict(q_heads=65536), dict(positions=0), dict(positions=p + 2), dict(axis_stride=-1), dict(q_heads=-1), dict(k_heads=-1),
           dict(q_heads=0, k_heads=0), dict(q=(0, 32, 16)), dict(q_out=(0, 32, 16)), dict(q=(p + 2, 32, 16)), dict(q_out=(p + 4098, 32, 16)),
           dict(q=(p + 1024, -32, 16)), dict(q_out=(p + 4096, 32, 0)), dict(q_out=(p + 4096, 16, 16)), dict(q_out=(p + 4096, 32, 8)),
           dict(q_out=(p + 1024, 64, 16)), dict(k_out=(0, 0, 0)), dict(k_out=(p + 8192, 0, 16))]
    bad += [{**cache, **kw} for kw in (dict(v_cache=0), dict(k_cache=0), dict(v=(0, 0, 0)), dict(slots=0), dict(slots=p + 20484), dict(block_size=0),
                                       dict(n_blocks=-1), dict(v_cache=p + 12288), dict(k_cache=p + 12290), dict(block_stride=16), dict(slot_stride=8),
                                       dict(slot_stride=-16), dict(k_heads=0))]
    for kw in bad:
        refused(E, r.apply, **{**good, **kw})
    backend.sync()
    assert (backend.get(data) == 0).all()
    r.apply(**{**good, "n_tokens": 0})  # no tokens are none
    r.close()


def check_bad_blocks(backend):
    """Blocks outside the cache, in the table and on the stack, give no slots."""
    check_slots(backend, "prompts", bad_ids=True)
    check_slots(backend, "step", bad_ids=True)


def check_more_tokens_than_64_bits_count(backend):
    """Segments of 2^64 tokens together: the sum does not wrap, and the first places are right."""
    most, left = 32767, 2 ** 64
    segments = [(2, 0, 0, 0)] + [(most, most, most, 1)] * ((left - 2) // most ** 3)
    left -= sum(t * h * w for t, h, w, _ in segments[1:]) + 2
    for t, h in ((most, most), (1, most)):
        segments.append((t, h, left // (t * h), 1))
        left -= t * h * segments[-1][2]
    segments.append((left, 0, 0, 0))
    assert len(segments) <= 1 << 20 and left > 0
    n, capacity = len(segments), 5000
    flat, seq = backend.put(np.array(segments, dtype=np.int32)), backend.put(np.array([0, n - 1, n], dtype=np.int32))
    positions, starts = backend.put(np.full((3, capacity), 77, dtype=np.int32)), backend.put(np.full(3, 77, dtype=np.int32))
    size = prep.token_positions_workspace(n)
    work = backend.put(np.zeros(size, dtype=np.uint8))
    prep.token_positions(backend.ptr(flat), n, backend.ptr(seq), 2, 0, 1, backend.ptr(positions), capacity, backend.ptr(starts), 0, backend.ptr(work), size,
                         stream=backend.stream)
    assert backend.get(starts).tolist() == [0, 2 ** 31 - 1, 2 ** 31 - 1]
    i = np.arange(capacity - 2)
    want = np.stack([np.append([0, 1], 2 + v) for v in (0 * i, i // most, i % most)])
    assert np.array_equal(backend.get(positions), want)


def check_slow_pairs(backend, adjacent=False):
    """sin of small angles (a = 1, b = 0), against the formula in extended precision, relative to itself: the angle is rounded when its parts
    become floats, when these are added, with the constant 2 pi and with the product, the series' terms and the result once each: 8 half steps
    of 2^-24; a frequency is held to 2^-63 of a turn, 2^-22 of one being the slowest here, and x^11 / 11! left out, 3e-9 of sin x."""
    d, base, places = 128, 1e6, np.array([1, -1, 2, 7, -50, 1000, 30000, -777777], dtype=np.int64)
    n, pairs = len(places), d // 2
    x = np.zeros((n, 1, d), dtype=np.float32)
    x[..., 0:d:2] = 1.0 if adjacent else 0.0
    if not adjacent:
        x[..., :pairs] = 1.0
    given, out = backend.put(x), backend.put(np.zeros_like(x))
    positions = backend.put(places.astype(np.int32))
    rotary = prep.Rotary(d, (pairs, 0, 0), base, "f32", pairing=int(adjacent))
    rotary.apply(n, backend.ptr(positions), n, q=(backend.ptr(given), d, d), q_out=(backend.ptr(out), d, d), q_heads=1, stream=backend.stream)
    got = backend.get(out)[:, 0].astype(np.longdouble)
    rotary.close()
    sine = got[:, 1::2] if adjacent else got[:, pairs:]
    angle = places[:, None].astype(np.longdouble) * np.array(oracle.frequencies((pairs, 0, 0), base, False, False))[None]
    small = np.abs(angle) <= np.pi / 4
    assert small.sum() > 200 and np.abs(angle).min() < 2e-6
    want = np.sin(angle)
    assert (np.abs(sine - want)[small] <= np.abs(want)[small] * (8 * ULP + 3e-9 + 2.0 ** -40)).all()


# ---- clips over several launches, given frequencies, segments of no sequence ------------------------------------------------

# (a launch takes 64 clips of a kind; those narrower than 6 pixels are of a kind of their own)
PATCHES_MORE = {
    "several_launches": ([(4 + i % 5, 4 + i % 3) for i in range(170)], [1] * 170, 4, 1, 1, "f16", True, 0, 0),
    # reductions of both axes by 2.25, 2.5, 2.81, 3 and 3.21: windows of 5, 6, 6, 7 and 7 samples
    "window_of_five": ([(225, 45)], [1], 2, 1, 1, "f32", True, 0, 100 * 20),
    "window_of_six_least": ([(225, 45), (45, 110)], [1, 1], 2, 1, 1, "f32", True, 0, 90 * 18),
    "window_of_six": ([(225, 45)], [2], 4, 1, 1, "f16", True, 0, 80 * 16),
    "window_of_seven_least": ([(240, 48)], [1], 8, 1, 2, "f32", True, 0, 80 * 16),
    "window_of_seven": ([(225, 45)], [1], 2, 1, 1, "f32", True, 0, 70 * 14),
    "several_launches_of_clips": ([(3 + i % 7, 9 - i % 4) for i in range(150)], [1 + i % 3 for i in range(150)], 3, 1, 2, "f32", False, 0, 0),
}

def check_more_patches(backend, name):
    PATCHES_LARGE[name] = (PATCHES_MORE | PATCHES_MIXED)[name]
    try:
        check_patches(backend, name)
    finally:
        del PATCHES_LARGE[name]


# many photographs with larger pictures between them, in launches of two kinds (a GPU's)
PATCHES_MIXED = {"large_mixed": ([(640, 480)] * 7 + [(1500, 1200)] + [(640, 480)] * 7, [1] * 15, 16, 2, 1, "f16", True, 0, 640 * 480)}

# frequencies in radians a place: negative, zero, whole turns, above a turn
FREQUENCIES = [0.0, -0.0, 1.0, -1.0, 0.3, -0.7, 1e-6, -1e-9, 2 * math.pi, -2 * math.pi, math.pi, 5.5, -6.2, 1e-3, -0.05, 2.0 ** -20]


def check_given_frequencies(backend, adjacent, dtype="f32"):
    """The base is not looked at, and a negative frequency turns the other way."""
    n, h, d, pairs = 12, 2, 40, len(FREQUENCIES)
    rng = np.random.default_rng(7)
    x = unpack(pack(rng.standard_normal((n, h, d)), dtype), dtype)
    positions = rng.integers(-2000, 2000, (3, n))
    positions[:, :2] = [[2 ** 30, -2 ** 31]] * 3
    sections = (5, 6, 5)
    given, out = backend.put(pack(x, dtype)), backend.put(pack(np.zeros_like(x), dtype))
    places = backend.put(positions.astype(np.int32))
    rotary = prep.Rotary(d, sections, float("nan"), dtype, pairing=int(adjacent), per_axis=True, frequencies=FREQUENCIES)
    rotary.apply(n, backend.ptr(places), n, q=(backend.ptr(given), h * d, d), q_out=(backend.ptr(out), h * d, d), q_heads=h, stream=backend.stream)
    got = unpack(backend.get(out), dtype)
    rotary.close()
    # the oracle's angle is a product of 64 bits, whose half step at 2^31 places of 2 pi is 2^-31 radians; the call's is off by 2^-31 of a turn
    extra = 2.0 ** -31 * (1 + 2 * math.pi)
    want = oracle.rotary(x, positions, oracle.pair_axes(sections, False), FREQUENCIES, adjacent, False)
    within(got, want, rotary_tolerance(x, pairs, adjacent) * (1 + extra / TRIG), dtype)
    assert np.array_equal(got[..., 2 * pairs:], x[..., 2 * pairs:])


def check_segments_of_no_sequence(backend, many):
    """Segments before the first sequence's and behind the last one's count for nothing, and bounds outside the list are its ends."""
    piece = [T(2), G(1, 2, 3), T(0), G(2, 3, 1, 4), T(1)]
    flat = piece * (1000 if many else 6)
    n = len(flat)
    for bounds in ([3, 3, 9, n - 4], [-7, 2, 5, n - 1], [1, n - 2, n, n + 50], [-3, -1, n + 1, n + 9], [n, n, n, n], [-9, -9, -9, -9]):
        clamped = np.clip(bounds, 0, n)
        first = [10, -3, 500]
        want, starts, nexts = oracle.token_positions([flat[a:b] for a, b in zip(clamped, clamped[1:])], first, 2)
        capacity = starts[-1] + 6
        segments, seq, base = backend.put(np.array(flat, dtype=np.int32)), backend.put(np.array(bounds, dtype=np.int32)), backend.put(np.array(first, dtype=np.int32))
        positions, token_starts, nxt = (backend.put(np.full(m, 77, dtype=np.int32)) for m in (3 * capacity, 4, 3))
        size = prep.token_positions_workspace(n)
        work = backend.put(np.full(size, 77, dtype=np.uint8))
        prep.token_positions(backend.ptr(segments), n, backend.ptr(seq), 3, backend.ptr(base), 2, backend.ptr(positions), capacity, backend.ptr(token_starts),
                             backend.ptr(nxt), backend.ptr(work), size, stream=backend.stream)
        full = np.zeros((3, capacity), dtype=np.int64)
        full[:, :starts[-1]] = want
        assert np.array_equal(backend.get(positions).reshape(3, capacity), full), bounds
        assert backend.get(token_starts).tolist() == starts and backend.get(nxt).tolist() == nexts, bounds
