"""The operators for packed batches of tokens on the GPU, against the oracle: the cases that the CPU build of the kernels
passes too, then larger ones, captured calls, the path from JPEG files, and a run of all of them together."""
import numpy as np
import pytest

import oracle as jpeg_oracle
import paper_2411_19114_amd as prep
import synth
import token_cases as cases
from oracle import tokens as oracle

pytestmark = pytest.mark.gpu


class Backend:
    def __init__(self):
        import torch
        self.torch = torch
        assert torch.cuda.is_available()

    @property
    def stream(self):
        return self.torch.cuda.current_stream().cuda_stream

    def put(self, a):
        a = np.ascontiguousarray(a)
        raw = self.torch.from_numpy(a.reshape(-1).view(np.uint8).copy()).cuda()
        if raw.numel() == 0:
            raw = self.torch.zeros(16, dtype=self.torch.uint8, device="cuda")
        return raw, a.shape, a.dtype

    def ptr(self, b):
        return b[0].data_ptr()

    def get(self, b):
        raw, shape, dtype = b
        return raw.cpu().numpy()[:int(np.prod(shape)) * dtype.itemsize].view(dtype).reshape(shape)

    def sync(self):
        self.torch.cuda.synchronize()


@pytest.fixture(scope="module")
def backend():
    return Backend()


@pytest.mark.parametrize("name", cases.PATCHES)
def test_patch_rows(backend, name):
    cases.check_patches(backend, name)
    cases.check_patches(backend, name, seed=1, out_pad=0, pitch_pad=0, lead=0)


@pytest.mark.parametrize("name", cases.PATCHES_LARGE)
def test_many_patch_rows(backend, name):
    cases.check_patches(backend, name)


@pytest.mark.parametrize("name", cases.ROTARY_LARGE)
def test_many_rotated_rows(backend, name):
    cases.check_rotary(backend, name)


@pytest.mark.parametrize("name", cases.POSITIONS)
def test_places(backend, name):
    cases.check_positions(backend, name)
    cases.check_positions(backend, name, workspace_pad=64, misaligned=1)


@pytest.mark.parametrize("name", cases.SLOTS)
def test_slots(backend, name):
    cases.check_slots(backend, name)


def test_bad_blocks(backend):
    cases.check_bad_blocks(backend)


@pytest.mark.parametrize("name", cases.ROTARY)
def test_rotary(backend, name):
    cases.check_rotary(backend, name)


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_gradient(backend, adjacent):
    cases.check_rotary_gradient(backend, adjacent)


def test_refusals(backend):
    cases.check_patch_refusals(backend)
    cases.check_packing_refusals(backend)
    cases.check_rotary_refusals(backend)


def test_a_device_that_is_not_there(backend):
    """An error, and the current device and the calls after it are as before."""
    torch = backend.torch
    x = torch.zeros(4096, dtype=torch.int64, device="cuda")
    p = x.data_ptr()
    params = prep.make_patch_params(4, 1, 1, "f32", cases.MEAN, cases.STD)
    cases.refused(prep.E_HIP, prep.patch_rows, 99, p, [0], [4], [4], [12], params, p + 4096, 10)
    cases.refused(prep.E_HIP, prep.token_positions, p, 1, p, 1, 0, 1, p + 4096, 8, p + 8192, 0, p + 16384, 1024, device=99)
    cases.refused(prep.E_HIP, prep.block_slots, 1, 4, 9, p, p + 64, p + 128, 4, p + 256, p + 512, 4, 4, p + 1024, 8, p + 2048, p + 2304, p + 2560, p + 2816,
                  p + 4096, 1024, device=99)
    assert torch.cuda.current_device() == 0
    torch.cuda.synchronize()
    cases.check_slots(backend, "step")


def test_two_streams_at_once(backend):
    """Calls that overlap on two streams, each with its own outputs and one rotary handle between them."""
    torch = backend.torch
    rng = np.random.default_rng(6)
    rotary = prep.Rotary(64, (16, 8, 8), 1e4, "f32")
    n, h = 4000, 4
    positions = rng.integers(0, 5000, (3, n)).astype(np.int32)
    x = [rng.standard_normal((n, h, 64)).astype(np.float32) for _ in range(2)]
    image = rng.integers(0, 256, (1, 300, 400, 3)).astype(np.uint8)
    params = prep.make_patch_params(16, 2, 1, "f32", cases.MEAN, cases.STD)
    places, src = torch.from_numpy(positions).cuda(), torch.from_numpy(image.reshape(-1)).cuda()
    given, out = [torch.from_numpy(v).cuda() for v in x], [torch.zeros((n, h, 64), device="cuda") for _ in range(2)]
    grid = prep.patch_grid(params, 400, 300)
    rows = grid[1] * grid[2]
    pixels = [torch.zeros((rows, 768), device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            rotary.apply(n, places.data_ptr(), n, q=(given[i].data_ptr(), h * 64, 64), q_out=(out[i].data_ptr(), h * 64, 64), q_heads=h, stream=s.cuda_stream)
            prep.patch_rows(0, src.data_ptr(), [0], [400], [300], [1200], params, pixels[i].data_ptr(), rows, stream=s.cuda_stream)
    torch.cuda.synchronize()
    axes, freqs = oracle.pair_axes((16, 8, 8), False), oracle.frequencies((16, 8, 8), 1e4, False, False)
    want_rows = oracle.patch_rows(image, grid[1] * 16, grid[2] * 16, 16, 2, 1, False, cases.MEAN, cases.STD)
    for i in range(2):
        v = x[i].astype(np.float64)
        cases.within(out[i].cpu().double().numpy(), oracle.rotary(v, positions, axes, freqs, False, False), cases.rotary_tolerance(v, 32, False), "f32")
        cases.within(pixels[i].cpu().double().numpy(), want_rows, cases.patch_tolerance(400, 300, grid[2] * 16, grid[1] * 16, False), "f32")
    rotary.close()


def test_another_stream(backend):
    """Work goes to the stream that is named, whatever the current one."""
    torch = backend.torch
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cases.check_patches(backend, "odd")
        cases.check_positions(backend, "merged")
        cases.check_slots(backend, "prompts")
        cases.check_rotary(backend, "store")


@pytest.mark.parametrize("dtype,antialias", [("bf16", True), ("f32", False)])
def test_patch_rows_of_jpeg_files(dtype, antialias):
    """The same rows as the oracle's, from the oracle's decoder; files that are refused have none, damaged ones zeros."""
    import torch
    rng = np.random.default_rng(8)
    sizes = [(97, 64), (33, 41), (240, 130), (64, 64), (80, 50)]
    files = [jpeg_oracle.encode(synth.gradient_noise_image(rng, w, h, 9.0), 88, mode, dri)[0]
             for (w, h), mode, dri in zip(sizes, (jpeg_oracle.MODE_420, jpeg_oracle.MODE_444, jpeg_oracle.MODE_420, jpeg_oracle.MODE_GRAY, jpeg_oracle.MODE_422),
                                          (0, 4, 8, 0, 0))]
    broken = bytearray(files[3])
    sos = broken.index(b"\xff\xda")
    del broken[sos + 40:-2]  # ends too early
    files[3] = bytes(broken)
    files[1] = b"\xff\xd8 not a picture \xff\xd9"
    blob, offsets = synth.pack(files)
    params = prep.make_patch_params(8, 2, 1, dtype, cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS if antialias else prep.FILTER_BILINEAR,
                                    max_pixels=120 * 120)
    pp = prep.Preprocessor(max_batch=len(files), max_width=256, max_height=256, max_bitstream_bytes=len(blob) + 64)
    row = 3 * 64
    resident = torch.from_numpy(np.frombuffer(bytes(blob), dtype=np.uint8).copy()).cuda()
    for device_bits in (0, resident.data_ptr()):
        out = torch.full((1000, row), -77.0, dtype={"bf16": torch.bfloat16, "f32": torch.float32}[dtype], device="cuda")
        starts = pp.decode_patches_batch(blob, offsets, params, out.data_ptr(), 1000, bitstreams_device_ptr=device_bits,
                                         stream=torch.cuda.current_stream().cuda_stream)
        status = pp.get_status(len(files))
        assert status[0] == status[2] == status[4] == 0 and status[1] in (prep.E_CORRUPT, prep.E_UNSUPPORTED) and status[3] == prep.E_CORRUPT
        got = out.cpu().double().numpy()
        at = 0
        for i, ((w, h), data) in enumerate(zip(sizes, files)):
            assert starts[i] == at
            if i == 1:
                continue
            oh, ow = oracle.patch_size(w, h, 8, 2, 0, 120 * 120)
            count = oh * ow // 64
            if i == 3:
                assert (got[at:at + count] == 0).all()
            else:
                _, rgb, _ = jpeg_oracle.decode(data)
                want = oracle.patch_rows(rgb[None], oh, ow, 8, 2, 1, antialias, cases.MEAN, cases.STD)
                # a decoded value may be one level off, and few are
                d = np.abs(got[at:at + count] - want)
                level = 1 / 255 / min(cases.STD)
                rounding = cases.HALF_STEP[dtype] * np.abs(want).max() + cases.patch_tolerance(w, h, ow, oh, antialias)
                assert d.max() <= level + rounding and (d > rounding).mean() < 0.01
            at += count
        assert starts[-1] == at and (got[at:] == -77).all()
    with pytest.raises(prep.PrepError) as e:
        pp.decode_patches_batch(blob, offsets, params, out.data_ptr(), starts[-1] - 1)
    assert e.value.code == prep.E_TOO_LARGE
    assert pp.decode_patches_batch(blob, offsets[:1], params, out.data_ptr(), 0) == [0]
    pp.close()


def test_captured_calls_follow_their_lengths(backend):
    """Places, slots and the rotation into the cache in one graph, replayed as the lengths on the GPU change, with other work between."""
    torch = backend.torch
    rng = np.random.default_rng(2)
    n, capacity, block, width, n_blocks, kh, d = 6, 96, 4, 16, 80, 2, 32
    i32 = dict(dtype=torch.int32, device="cuda")
    segments, seq = torch.zeros((n, 4), **i32), torch.arange(n + 1, **i32)
    cached, fresh = torch.zeros(n, **i32), torch.zeros(n, **i32)
    positions, starts, nexts = torch.zeros((3, capacity), **i32), torch.zeros(n + 1, **i32), torch.zeros(n, **i32)
    table, lengths, status = torch.full((n, width), -1, **i32), torch.zeros(n, **i32), torch.zeros(n, **i32)
    stack = torch.from_numpy(rng.permutation(n_blocks).astype(np.int32)).cuda()
    counts = [torch.full((1,), n_blocks, **i32), torch.zeros(1, **i32)]
    slots, token_starts = torch.zeros(capacity, dtype=torch.int64, device="cuda"), torch.zeros(n + 1, **i32)
    work = [torch.zeros(1024, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = (torch.zeros((capacity, kh, d), device="cuda") for _ in range(2))
    caches = [torch.zeros((n_blocks, block, kh, d), device="cuda") for _ in range(2)]
    rotary = prep.Rotary(d, (8, 4, 4), 1e4, "f32")

    def step():
        s = torch.cuda.current_stream().cuda_stream
        prep.token_positions(segments.data_ptr(), n, seq.data_ptr(), n, cached.data_ptr(), 1, positions.data_ptr(), capacity, starts.data_ptr(),
                             nexts.data_ptr(), work[0].data_ptr(), 1024, stream=s)
        prep.block_slots(n, block, n_blocks, cached.data_ptr(), fresh.data_ptr(), stack.data_ptr(), n_blocks, counts[0].data_ptr(), table.data_ptr(),
                         width, width, slots.data_ptr(), capacity, token_starts.data_ptr(), lengths.data_ptr(), status.data_ptr(),
                         counts[1].data_ptr(), work[1].data_ptr(), 1024, stream=s)
        rotary.apply(capacity, positions.data_ptr(), capacity, k=(k.data_ptr(), kh * d, d), k_heads=kh, v=(v.data_ptr(), kh * d, d),
                     k_cache=caches[0].data_ptr(), v_cache=caches[1].data_ptr(), n_blocks=n_blocks, block_size=block, block_stride=block * kh * d,
                     slot_stride=kh * d, cache_head_stride=d, slots=slots.data_ptr(), stream=s)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held = np.zeros(n, dtype=int)
    on_stack = stack.cpu().numpy().tolist()
    tables = np.full((n, width), -1, dtype=np.int32)
    want = [np.zeros((n_blocks * block, kh, d)) for _ in range(2)]
    freqs, axes = oracle.frequencies((8, 4, 4), 1e4, False, False), oracle.pair_axes((8, 4, 4), False)
    for _ in range(4):
        new = rng.integers(0, 17, n)
        kk, vv = (rng.standard_normal((capacity, kh, d)).astype(np.float32) for _ in range(2))
        segments[:, 0] = torch.from_numpy(new.astype(np.int32)).cuda()
        cached.copy_(torch.from_numpy(held.astype(np.int32)))
        fresh.copy_(torch.from_numpy(new.astype(np.int32)))
        k.copy_(torch.from_numpy(kk))
        v.copy_(torch.from_numpy(vv))
        graph.replay()
        torch.cuda.synchronize()
        spot, tables, first, lens, stat, left = oracle.block_slots(held, new, block, n_blocks, np.array(on_stack, dtype=np.int32), tables, capacity)
        assert (stat == 0).all() and np.array_equal(slots.cpu().numpy(), spot) and np.array_equal(table.cpu().numpy(), tables)
        assert lengths.cpu().numpy().tolist() == lens.tolist() and counts[1].item() == left and token_starts.cpu().numpy().tolist() == first.tolist()
        places, first2, _ = oracle.token_positions([[(int(m), 0, 0, 0)] for m in new], held.tolist(), 1)
        full = np.zeros((3, capacity), dtype=np.int64)
        full[:, :places.shape[1]] = places
        assert np.array_equal(positions.cpu().numpy(), full) and first2 == first.tolist()
        turned = oracle.rotary(kk.astype(np.float64), full, axes, freqs, False, False)
        real = np.flatnonzero(spot >= 0)
        want[0][spot[real]], want[1][spot[real]] = turned[real], vv[real]
        tolerance = cases.rotary_tolerance(np.abs(kk.astype(np.float64)).max() * np.ones((1, 1, d)), 16, False)
        cases.within(caches[0].cpu().double().numpy().reshape(-1, kh, d), want[0], tolerance, "f32")
        assert np.array_equal(caches[1].cpu().numpy().reshape(-1, kh, d), want[1].astype(np.float32))
        del on_stack[left:]
        counts[0].copy_(counts[1])
        held += new
        torch.randn(1000, device="cuda").sum().item()  # eager work between the replays
    rotary.close()


def test_captured_patch_rows_and_backward_rotation(backend):
    """One graph of both, replayed on new contents of the same buffers with eager work between, against the oracle and an eager call."""
    torch = backend.torch
    rng = np.random.default_rng(9)
    w, h, n, heads, d = 200, 150, 300, 3, 64
    params = prep.make_patch_params(14, 2, 2, "f32", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, max_pixels=120 * 120)
    grid = prep.patch_grid(params, w, h, 3)
    rows = grid[0] * grid[1] * grid[2]
    src = torch.zeros(3 * h * w * 3, dtype=torch.uint8, device="cuda")
    pixels, gradient, out = torch.zeros((rows, 1176), device="cuda"), torch.zeros((n, heads, d), device="cuda"), torch.zeros((n, heads, d), device="cuda")
    places = torch.zeros((3, n), dtype=torch.int32, device="cuda")
    rotary = prep.Rotary(d, (12, 10, 10), 1e4, "f32")

    def both(pixels, out):
        s = torch.cuda.current_stream().cuda_stream
        prep.patch_rows(0, src.data_ptr(), [0], [w], [h], [3 * w], params, pixels.data_ptr(), rows, frames=[3], frame_strides=[3 * w * h], stream=s)
        rotary.apply(n, places.data_ptr(), n, q=(gradient.data_ptr(), heads * d, d), q_out=(out.data_ptr(), heads * d, d), q_heads=heads, inverse=True, stream=s)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(pixels, out)
    axes, freqs = oracle.pair_axes((12, 10, 10), False), oracle.frequencies((12, 10, 10), 1e4, False, False)
    for _ in range(4):
        clip = cases.picture(rng, (3, h, w, 3))
        g = rng.standard_normal((n, heads, d)).astype(np.float32)
        p = rng.integers(0, 9000, (3, n)).astype(np.int32)
        src.copy_(torch.from_numpy(clip.reshape(-1)))
        gradient.copy_(torch.from_numpy(g))
        places.copy_(torch.from_numpy(p))
        graph.replay()
        eager = torch.zeros_like(pixels), torch.zeros_like(out)
        both(*eager)
        torch.cuda.synchronize()
        assert torch.equal(eager[0], pixels) and torch.equal(eager[1], out)
        want = oracle.patch_rows(clip, grid[1] * 14, grid[2] * 14, 14, 2, 2, True, cases.MEAN, cases.STD)
        cases.within(pixels.cpu().double().numpy(), want, cases.patch_tolerance(w, h, grid[2] * 14, grid[1] * 14, True), "f32")
        v = g.astype(np.float64)
        cases.within(out.cpu().double().numpy(), oracle.rotary(v, p, axes, freqs, False, True), cases.rotary_tolerance(v, 32, False), "f32")
    rotary.close()


def test_from_files_to_the_cache(backend):
    """A step of a model that reads pictures, without the model: files to patch rows, the encoder's places and rotation, then the places,
    slots and rotation into the cache of prompts that hold the pictures' merged tokens."""
    torch = backend.torch
    rng = np.random.default_rng(12)
    patch, merge, heads, d = 8, 2, 2, 32
    sizes = [(70, 50), (48, 96)]
    files = [jpeg_oracle.encode(synth.gradient_noise_image(rng, w, h, 9.0), 90, jpeg_oracle.MODE_444, 0)[0] for w, h in sizes]
    blob, offsets = synth.pack(files)
    params = prep.make_patch_params(patch, merge, 1, "f32", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS)
    grids = [prep.patch_grid(params, w, h) for w, h in sizes]
    rows = sum(a * b * c for a, b, c in grids)
    s = torch.cuda.current_stream().cuda_stream
    pp = prep.Preprocessor(max_batch=2, max_width=128, max_height=128, max_bitstream_bytes=len(blob))
    pixels = torch.zeros((rows, 3 * patch * patch), device="cuda")
    assert pp.decode_patches_batch(blob, offsets, params, pixels.data_ptr(), rows, stream=s)[-1] == rows
    # the encoder's queries and keys from the rows: a projection of the test's own
    project = torch.from_numpy(rng.standard_normal((3 * patch * patch, 2 * heads * d)).astype(np.float32) / 14).cuda()
    qk = (pixels @ project).reshape(rows, 2 * heads, d).contiguous()
    i32 = dict(dtype=torch.int32, device="cuda")

    def places(sequences, first, m):
        flat = torch.tensor([x for q in sequences for x in q], **i32).reshape(-1, 4)
        bounds = torch.tensor(np.cumsum([0] + [len(q) for q in sequences]), **i32)
        total = len(oracle.token_positions(sequences, first, m)[0][0])
        out, starts, nexts = torch.zeros((3, total), **i32), torch.zeros(len(sequences) + 1, **i32), torch.zeros(len(sequences), **i32)
        size = prep.token_positions_workspace(len(flat))
        work, base = torch.zeros(size, dtype=torch.uint8, device="cuda"), torch.tensor(first, **i32)
        prep.token_positions(flat.data_ptr(), len(flat), bounds.data_ptr(), len(sequences), base.data_ptr(), m, out.data_ptr(), total, starts.data_ptr(),
                             nexts.data_ptr(), work.data_ptr(), size, stream=s)
        return out, starts, nexts

    seen, _, _ = places([[(1, h, w, 1)] for _, h, w in grids], [0, 0], merge)
    encoder = prep.Rotary(d, (0, 8, 8), 1e4, "f32", per_axis=True)
    q_out = torch.zeros((rows, heads, d), device="cuda")
    base = qk.data_ptr()
    encoder.apply(rows, seen.data_ptr(), rows, q=(base, 2 * heads * d, d), q_out=(q_out.data_ptr(), heads * d, d), q_heads=heads,
                  k=(base + 4 * heads * d, 2 * heads * d, d), k_out=(base + 4 * heads * d, 2 * heads * d, d), k_heads=heads, stream=s)
    # two prompts with the merged pictures between words
    sequences = [[(3, 0, 0, 0), (1, grids[0][1] // merge, grids[0][2] // merge, 1), (2, 0, 0, 0)], [(1, grids[1][1] // merge, grids[1][2] // merge, 1), (4, 0, 0, 0)]]
    spots, starts, nexts = places(sequences, [0, 0], 1)
    want_places, want_starts, want_next = oracle.token_positions(sequences, [0, 0], 1)
    n = want_places.shape[1]
    assert starts.tolist() == want_starts and nexts.tolist() == want_next and np.array_equal(spots.cpu().numpy(), want_places)
    fresh = torch.tensor(np.diff(want_starts), **i32)
    cached = torch.zeros(2, **i32)
    block, width, n_blocks = 4, 32, 40
    table, stack = torch.zeros((2, width), **i32), torch.arange(n_blocks, **i32)
    count, left, lengths, status = torch.full((1,), n_blocks, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32), torch.zeros(2, **i32)
    slots = torch.zeros(n, dtype=torch.int64, device="cuda")
    size = prep.block_slots_workspace(2)
    work = torch.zeros(size, dtype=torch.uint8, device="cuda")
    prep.block_slots(2, block, n_blocks, cached.data_ptr(), fresh.data_ptr(), stack.data_ptr(), n_blocks, count.data_ptr(), table.data_ptr(), width, width,
                     slots.data_ptr(), n, starts.data_ptr(), lengths.data_ptr(), status.data_ptr(), left.data_ptr(), work.data_ptr(), size, stream=s)
    kv = torch.from_numpy(rng.standard_normal((n, 2, d)).astype(np.float32)).cuda()
    caches = torch.zeros((2, n_blocks, block, 1, d), device="cuda")
    model = prep.Rotary(d, (6, 5, 5), 1e4, "f32")
    model.apply(n, spots.data_ptr(), n, k=(kv.data_ptr(), 2 * d, d), k_heads=1, v=(kv.data_ptr() + 4 * d, 2 * d, d), k_cache=caches[0].data_ptr(),
                v_cache=caches[1].data_ptr(), n_blocks=n_blocks, block_size=block, block_stride=block * d, slot_stride=d, cache_head_stride=d,
                slots=slots.data_ptr(), stream=s)
    torch.cuda.synchronize()
    # patch rows: those of the decoded pictures (a level where the decoder is one off)
    level = 1 / 255 / min(cases.STD)
    at = 0
    want_rows = []
    for (w, h), data, grid in zip(sizes, files, grids):
        _, rgb, _ = jpeg_oracle.decode(data)
        want_rows.append(oracle.patch_rows(rgb[None], grid[1] * patch, grid[2] * patch, patch, merge, 1, True, cases.MEAN, cases.STD))
        at += len(want_rows[-1])
    assert np.abs(pixels.cpu().double().numpy() - np.concatenate(want_rows)).max() <= level + 1e-5
    # the encoder's rotation of what the test's own projection gave
    given = (pixels @ project).reshape(rows, 2 * heads, d).cpu().double().numpy()
    want_seen, _, _ = oracle.token_positions([[(1, h, w, 1)] for _, h, w in grids], [0, 0], merge)
    axes, freqs = oracle.pair_axes((0, 8, 8), False), oracle.frequencies((0, 8, 8), 1e4, False, True)
    turned = oracle.rotary(given, want_seen, axes, freqs, False, False)
    cases.within(q_out.cpu().double().numpy(), turned[:, :heads], cases.rotary_tolerance(given[:, :heads], 16, False), "f32")
    cases.within(qk[:, heads:].cpu().double().numpy(), turned[:, heads:], cases.rotary_tolerance(given[:, heads:], 16, False), "f32")
    # the cache: every token's key and value where the block table says
    axes, freqs = oracle.pair_axes((6, 5, 5), False), oracle.frequencies((6, 5, 5), 1e4, False, False)
    key = kv.cpu().double().numpy()
    turned = oracle.rotary(key[:, :1], want_places, axes, freqs, False, False)
    assert status.tolist() == [0, 0] and lengths.tolist() == np.diff(want_starts).tolist()
    blocks = table.cpu().numpy()
    held = caches.cpu().double().numpy()
    for i in range(2):
        for j in range(want_starts[i + 1] - want_starts[i]):
            t = want_starts[i] + j
            b = blocks[i, j // block]
            cases.within(held[0, b, j % block], turned[t], cases.rotary_tolerance(key[t:t + 1, :1], 16, False)[0], "f32")
            assert np.array_equal(held[1, b, j % block, 0], key[t, 1])
    assert left.item() == n_blocks - sum(-(-int(f) // block) for f in np.diff(want_starts))
    pp.close()
    encoder.close()
    model.close()
