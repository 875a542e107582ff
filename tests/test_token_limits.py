"""Calls of the operators for packed batches of tokens whose sizes come near what 32 bits hold, without a GPU: their sources compiled by
g++, a few workgroups of each launch run on buffers of address space of which few pages are touched."""
import ctypes as C
import mmap
import os
import subprocess

import numpy as np
import pytest

import emul
import paper_2411_19114_amd.binding as prep
import token_cases as cases
from oracle import tokens as oracle


class Library:
    def __init__(self, path):
        self.lib = C.CDLL(path)

    def want(self, groups=()):
        self.lib.some_workgroups_want((C.c_uint64 * len(groups))(*groups), len(groups))

    def launches(self):
        """(workgroups before it, workgroups, threads) of each launch since want()."""
        out, got = (C.c_uint64 * 3)(), []
        for i in range(self.lib.some_workgroups_launch(1 << 30, out)):
            self.lib.some_workgroups_launch(i, out)
            got.append(tuple(out))
        return got


def _build(where, source, rest=""):
    path = str(where / (source + ".so"))
    (where / (source + ".cpp")).write_text(f'#include "some_workgroups.h"\n#include "{os.path.join(emul.CSRC, source)}"\n{rest}\n')
    subprocess.run(["g++", "-std=c++20", "-O1", "-pthread", "-fPIC", "-shared", "-I", emul.EMU, "-I", emul.CSRC, "-include",
                    os.path.join(emul.EMU, "more_hip.h"), str(where / (source + ".cpp")), "-o", path], check=True)
    return Library(path)


@pytest.fixture(scope="module")
def rotary(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("rotary"), "rotary.hip")


@pytest.fixture(scope="module")
def patches(tmp_path_factory):
    return _build(tmp_path_factory.mktemp("patches"), "patches.hip", "int prep::decode_batch(prep_handle *, const uint8_t *, const uint8_t *, const "
                  "uint64_t *, int32_t, OutputStage *, hipStream_t) { return PREP_E_INVALID_ARG; }")


class Sparse:
    """Zeros, of which only what is touched takes memory."""

    def __init__(self, size):
        self.map = mmap.mmap(-1, size, flags=mmap.MAP_PRIVATE | mmap.MAP_ANONYMOUS | 0x4000)  # MAP_NORESERVE
        self.bytes = np.frombuffer(self.map, dtype=np.uint8)
        self.ptr = self.bytes.ctypes.data


def _patch_rows(library, params, src, w, h, pitch, out, rows):
    starts = (C.c_int64 * 2)()
    rc = library.lib.prep_patch_rows(0, C.c_void_p(src), prep._packed("Q", [0]), prep._packed("i", [w]), prep._packed("i", [h]), prep._packed("i", [pitch]),
                                     None, None, 1, C.byref(params), C.c_void_p(out), C.c_int64(0), C.c_int64(rows), starts, None)
    return rc, list(starts)


def place_of_row(row, cols, merge):
    """(line, column) of patches of row `row` of a frame whose lines of patches come in windows of merge x merge."""
    band, r = divmod(row, merge * cols)
    window, r = divmod(r, merge * merge)
    return band * merge + r // merge, window * merge + r % merge


@pytest.mark.parametrize("side,merge", [(46368, 2), (65520, 5)])
def test_frames_of_more_than_2_31_pixels(patches, side, merge):
    """Rows of an enlarged still: those around pixel 2^31 of the rows' order, and the first and the last."""
    w, patch = 16, 16
    params = prep.make_patch_params(patch, merge, 1, "bf16", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, min_pixels=side * side)
    cols = side // patch
    rows, area = cols * cols, patch * patch
    assert rows * area > 2 ** 31
    picture = cases.picture(np.random.default_rng(4), (w, w, 3))
    # (as much room below the rows as a wrapped index reaches)
    row_bytes = 3 * area * 2
    below = 2 ** 31 * 6 + (1 << 20)
    out = Sparse(below + rows * row_bytes)
    looked_at = [0, 2 ** 31 // area - 1, 2 ** 31 // area, 2 ** 31 // area + 1, rows - 1]  # (256 pixels are a workgroup's and a row's)
    patches.want(looked_at)
    rc, starts = _patch_rows(patches, params, picture.ctypes.data, w, w, 3 * w, out.ptr + below, rows)
    assert rc == 0 and starts == [0, rows]
    weights = enlarging_weights(w, side)
    for row in looked_at:
        y, x = place_of_row(row, cols, merge)
        wy, wx = weights(range(y * patch, (y + 1) * patch)), weights(range(x * patch, (x + 1) * patch))
        v = np.stack([wy @ picture[..., c].astype(np.float64) @ wx.T for c in range(3)])
        want = ((v / 255 - np.array(cases.MEAN)[:, None, None]) / np.array(cases.STD)[:, None, None]).ravel()
        at = below + row * row_bytes
        got = cases.unpack(out.bytes[at:at + row_bytes].view(np.uint16), "bf16")
        cases.within(got, want, cases.patch_tolerance(w, w, side, side, True), "bf16")


def enlarging_weights(size, out):
    def rows(which):
        m = np.zeros((len(which), size))
        for k, i in enumerate(which):
            centre = (i + 0.5) * size / out - 0.5
            low = int(np.floor(centre))
            m[k, min(max(low, 0), size - 1)] += 1 - (centre - low)
            m[k, min(max(low + 1, 0), size - 1)] += centre - low
        return m
    return rows


@pytest.mark.parametrize("h", [26, 70])
@pytest.mark.parametrize("pitch", [3 * 40, 2 ** 26 + 128, 2 ** 27 + 64, 2 ** 30, 2 ** 31 - 1])
def test_rows_far_apart(patches, pitch, h):
    """Rows whose distance times the rows under a tile passes 32 bits."""
    w, patch, most = 40, 13, 0 if h == 26 else 26 * 26  # (near the picture's size, or reduced, so that a tile has many rows)
    params = prep.make_patch_params(patch, 1, 1, "f32", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, max_pixels=most)
    oh, ow = oracle.patch_size(w, h, patch, 1, 0, most)
    picture = cases.picture(np.random.default_rng(5), (h, w, 3))
    src = Sparse(pitch * (h - 1) + 3 * w)
    for y in range(h):
        src.bytes[y * pitch:y * pitch + 3 * w] = picture[y].ravel()
    want = oracle.patch_rows(picture[None], oh, ow, patch, 1, 1, True, cases.MEAN, cases.STD)
    out = np.zeros(want.shape, dtype=np.float32)
    patches.want(range(64))
    rc, starts = _patch_rows(patches, params, src.ptr, w, h, pitch, out.ctypes.data, len(want))
    assert rc == 0 and starts == [0, len(want)] and patches.launches()[-1][0] + patches.launches()[-1][1] <= 64
    cases.within(out.astype(np.float64), want, cases.patch_tolerance(w, h, ow, oh, True), "f32")


MOST = 2 ** 32 - 1  # work-items of a launch along an axis, by HIP's documentation


def in_launches_that_fit(launches):
    """Launches follow one another without gaps and each has a size that HIP takes."""
    at = 0
    for before, groups, threads in launches:
        assert before == at and 0 < groups and groups * threads <= MOST, launches
        at += groups
    return at


@pytest.mark.parametrize("frames,group", [(1, 2), (3, 1)])
def test_more_pixels_than_a_launch_has_work_items(patches, frames, group):
    """65 520 x 65 520 pixels in two slots or three frames: rows at the seams of the launches, and the last."""
    w, patch, side = 16, 16, 65520
    params = prep.make_patch_params(patch, 1, group, "bf16", cases.MEAN, cases.STD, prep.FILTER_BILINEAR, min_pixels=side * side)
    cols = side // patch
    rows, area = cols * cols, patch * patch
    picture = cases.picture(np.random.default_rng(6), (frames, w, w, 3))
    out = Sparse(3 * area * 2 * group * rows * (-(-frames // group)))
    total = rows * frames * group
    looked_at = [0, rows, MOST // 256 - 1, MOST // 256, 2 * (MOST // 256), total - 1]  # (a workgroup has the 256 pixels of a patch)
    looked_at = [r for r in looked_at if r < total]
    patches.want(looked_at)
    starts = (C.c_int64 * 2)()
    rc = patches.lib.prep_patch_rows(0, C.c_void_p(picture.ctypes.data), prep._packed("Q", [0]), prep._packed("i", [w]), prep._packed("i", [w]),
                                     prep._packed("i", [3 * w]), prep._packed("i", [frames]), prep._packed("Q", [3 * w * w]), 1, C.byref(params),
                                     C.c_void_p(out.ptr), C.c_int64(0), C.c_int64(2 ** 40), starts, None)
    assert rc == 0 and list(starts) == [0, rows * -(-frames // group)]
    assert in_launches_that_fit(patches.launches()) == total
    weights = enlarging_weights(w, side)
    values = out.bytes.view(np.uint16).reshape(-1, 3, group, area)
    for r in looked_at:
        slot, row = divmod(r, rows)
        y, x = divmod(row, cols)
        wy, wx = weights(range(y * patch, (y + 1) * patch)), weights(range(x * patch, (x + 1) * patch))
        v = np.stack([wy @ picture[min(slot, frames - 1), ..., c].astype(np.float64) @ wx.T for c in range(3)])
        want = ((v / 255 - np.array(cases.MEAN)[:, None, None]) / np.array(cases.STD)[:, None, None]).reshape(3, area)
        cases.within(cases.unpack(values[slot // group * rows + row, :, slot % group], "bf16"), want, cases.patch_tolerance(w, w, side, side, False), "bf16")


def test_clips_of_more_tiles_than_a_launch_has_work_items(patches):
    """Frames in tiles, 512 threads each: launches whose sizes HIP takes, one after another."""
    params = prep.make_patch_params(16, 1, 1, "f16", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, max_pixels=8000 * 2500)
    w, h, frames = 20000, 6000, 4000
    rows = np.prod(prep.patch_grid(params, w, h, frames))
    starts = (C.c_int64 * 2)()
    patches.want()
    rc = patches.lib.prep_patch_rows(0, C.c_void_p(4096), prep._packed("Q", [0]), prep._packed("i", [w]), prep._packed("i", [h]), prep._packed("i", [3 * w]),
                                     prep._packed("i", [frames]), prep._packed("Q", [3 * w * h]), 1, C.byref(params), C.c_void_p(4096), C.c_int64(0),
                                     C.c_int64(2 ** 50), starts, None)
    assert rc == 0 and list(starts) == [0, rows]
    assert in_launches_that_fit(patches.launches()) * 512 > MOST


def _rotary(library, head_dim, pairs, dtype):
    h = C.c_void_p()
    cfg = prep.RotaryConfig(0, head_dim, (C.c_int32 * 3)(pairs, 0, 0), {"f32": prep.F32, "bf16": prep.BF16}[dtype], 0, 0, 0, 0, 1e4, None)
    assert library.lib.prep_rotary_create(C.byref(h), C.byref(cfg)) == 0
    return h


@pytest.mark.parametrize("head_dim,pairs,dtype", [(2, 1, "bf16"), (32, 16, "f32")])
def test_more_rows_than_a_launch_has_work_items(rotary, head_dim, pairs, dtype):
    """One head of many tokens, a thread a pair and rows in 16 bytes: tokens at the seams of the launches, and the last."""
    n = 2 ** 31 - 1
    size = 2 if dtype == "bf16" else 4
    q, out, positions = Sparse(n * head_dim * size), Sparse(n * head_dim * size), Sparse(n * 4)
    handle = _rotary(rotary, head_dim, pairs, dtype)

    def call():
        return rotary.lib.prep_rotary_apply(handle, prep._ROTARY_ARGS.pack(
            n, positions.ptr, 0, q.ptr, head_dim, head_dim, out.ptr, head_dim, head_dim, *[0] * 9, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0), None)

    rotary.want()
    assert call() == 0
    launches = rotary.launches()
    groups = in_launches_that_fit(launches)
    assert len(launches) > 1
    step = next(s for s in range(1, 1025) if -(-n // s) == groups)  # tokens of a workgroup
    seams = [before for before, _, _ in launches] + [groups - 1]
    tokens = sorted({t for s in seams for t in (s * step - 1, s * step, min(s * step + step, n) - 1) if 0 <= t < n})
    rng = np.random.default_rng(3)
    x = cases.unpack(cases.pack(rng.standard_normal((len(tokens), 1, head_dim)), dtype), dtype)
    places = rng.integers(0, 2 ** 31, len(tokens))
    given, taken = (b.bytes.view(cases.NUMPY[dtype]).reshape(n, head_dim) for b in (q, out))
    given[tokens] = cases.pack(x[:, 0], dtype)
    positions.bytes.view(np.int32)[tokens] = places
    rotary.want([t // step for t in tokens])
    assert call() == 0
    rotary.lib.prep_rotary_destroy(handle)
    want = oracle.rotary(x, np.stack([places] * 3), [0] * pairs, oracle.frequencies((pairs, 0, 0), 1e4, False, False), False, False)
    cases.within(cases.unpack(taken[tokens], dtype), want[:, 0], cases.rotary_tolerance(x, pairs, False)[:, 0], dtype)


@pytest.mark.parametrize("short", ["rgb_offsets", "heights", "pitches", "frames", "frame_strides"])
def test_lists_of_different_lengths(short, monkeypatch):
    """The binding refuses them: the call would read behind the shorter one."""
    def never(*_):
        raise AssertionError("called")

    monkeypatch.setattr(prep, "_lib", type("Library", (), {"prep_patch_rows": never, "prep_strerror": lambda *_: b""})())
    lists = {"rgb_offsets": [0, 768], "widths": [16, 16], "heights": [16, 16], "pitches": [48, 48], "frames": [1, 1], "frame_strides": [768, 768]}
    lists[short] = lists[short][:1]
    params = prep.make_patch_params(16, 1, 1, "f32", cases.MEAN, cases.STD)
    cases.refused(prep.E_INVALID_ARG, prep.patch_rows, 0, 4096, params=params, out_ptr=8192, out_rows=2, **lists)


def test_more_rows_than_64_bits_count(patches):
    """2^24 + 9 clips of nearly 2^39 rows each are too many for any output, and nothing is enqueued."""
    n, frames = 2 ** 24 + 9, 2 ** 31 - 1
    params = prep.make_patch_params(1, 1, 1, "bf16", cases.MEAN, cases.STD)
    side, stride = np.full(n, 16, dtype=np.int32), np.full(n, 48 * 16, dtype=np.uint64)
    arrays = [np.zeros(n, dtype=np.uint64), side, side, np.full(n, 48, dtype=np.int32), np.full(n, frames, dtype=np.int32), stride]
    starts = np.zeros(n + 1, dtype=np.int64)
    assert n * frames * 256 > 2 ** 63
    patches.want()
    rc = patches.lib.prep_patch_rows(0, C.c_void_p(4096), *[C.c_void_p(a.ctypes.data) for a in arrays], n, C.byref(params), C.c_void_p(4096), C.c_int64(0),
                                     C.c_int64(2 ** 50), C.c_void_p(starts.ctypes.data), None)
    assert rc == prep.E_TOO_LARGE and patches.launches() == []
    assert (np.diff(starts) >= 0).all() and starts[-1] == 2 ** 63 - 1


@pytest.mark.parametrize("photographs,large,threads", [(30, 0, [256]), (30, 1, [256, 512]), (4, 1, [512]), (0, 2, [512]), (200, 3, [256] * 4 + [512])])
def test_large_pictures_among_photographs(patches, photographs, large, threads):
    """Many photographs keep the kernel for tiles with small windows (256 threads) when a picture that is reduced comes with them."""
    n = photographs + large
    sizes = [(4000, 3000) if i < large else (480, 360) for i in range(n)]
    params = prep.make_patch_params(16, 2, 1, "f16", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, max_pixels=1 << 20)
    starts = (C.c_int64 * (n + 1))()
    patches.want()
    rc = patches.lib.prep_patch_rows(0, C.c_void_p(4096), prep._packed("Q", [0] * n), prep._packed("i", [w for w, _ in sizes]), prep._packed("i", [h for _, h in sizes]),
                                     prep._packed("i", [3 * w for w, _ in sizes]), None, None, n, C.byref(params), C.c_void_p(4096), C.c_int64(0), C.c_int64(2 ** 30), starts, None)
    assert rc == 0 and [t for _, _, t in patches.launches()] == threads


def test_more_tiles_than_a_launch_counts(patches):
    """A frame of a column of 80 pixels has two strips of tiles: 2^31 - 1 frames have more of them than 32 bits count, and go pixel by pixel."""
    frames, w, h = 2 ** 31 - 1, 6, 480
    params = prep.make_patch_params(1, 1, 1, "bf16", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, max_pixels=80)
    assert prep.patch_grid(params, w, h, frames) == (frames, 80, 1)
    starts = (C.c_int64 * 2)()
    patches.want()
    rc = patches.lib.prep_patch_rows(0, C.c_void_p(4096), prep._packed("Q", [0]), prep._packed("i", [w]), prep._packed("i", [h]), prep._packed("i", [3 * w]),
                                     prep._packed("i", [frames]), prep._packed("Q", [3 * w * h]), 1, C.byref(params), C.c_void_p(4096), C.c_int64(0),
                                     C.c_int64(2 ** 50), starts, None)
    assert rc == 0 and list(starts) == [0, 80 * frames]
    assert in_launches_that_fit(patches.launches()) == -(-80 * frames // 256)
