"""What is timed of the operators that bring images, video and text into a language model's batch: patch rows from
decoded frames, positions with three axes, rotary embedding by them (with its inverse, and with the store into a paged
cache), and block tables with slot maps from request lengths.

`own` chooses between the framework's calls and the same operators in plain torch operations.
"""
import math

import numpy as np
import torch

own = False

MEAN, STD = (0.485, 0.456, 0.406), (0.229, 0.224, 0.225)
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # a request with one small picture, served by itself
        _patches("patches_one", 1, (256, 256), (256, 256), 1, 14, 2, 2, "bf16", "antialias"),
        # a batch of photographs of all sizes for a vision encoder, at their own sizes
        _patches("patches_photos_32", 32, (300, 640), (250, 500), 1, 16, 2, 1, "f16", "antialias"),
        # a full-HD clip reduced to about 400 000 pixels a frame, two frames a patch
        _patches("patches_clip_hd", 1, (1920, 1920), (1080, 1080), 48, 14, 2, 2, "bf16", "antialias", most=512 * 784),
        # frames of a training set read with the two-tap filter, fp32
        _patches("patches_train_64", 64, (480, 640), (360, 480), 1, 16, 1, 1, "f32", "bilinear", most=384 * 384),
        # one step of 64 sequences, a token each
        _positions("positions_step", 64, 64, "step", 1),
        # prompts with pictures and clips between pieces of text
        _positions("positions_prompts", 256, 400000, "mixed", 1),
        # one step of 48 sequences: rotate, and store k and v in the cache
        _rotary("rotary_step", 48, 32, 8, 128, (16, 24, 24), "bf16", "halves", "blocks", 500000.0, 65536, store=True, slots=32768),
        # prompts of 8192 tokens with images, stored in the cache
        _rotary("rotary_prompts", 8192, 28, 4, 128, (16, 24, 24), "bf16", "halves", "blocks", 1000000.0, 32768, store=True, slots=16384),
        # a vision encoder's patches: two axes, q and k inside a fused projection, odd number of tokens
        _rotary("rotary_patches", 19321, 16, 16, 80, (0, 20, 20), "f16", "halves", "blocks", 10000.0, 140, fused=True, ladder="axis"),
        # the backward pass of a training step in fp32, adjacent pairs
        _rotary("rotary_gradient", 16384, 32, 8, 64, (12, 10, 10), "f32", "adjacent", "interleaved", 10000.0, 16384, inverse=True),
        # one step of 128 requests, a token each, some of which begin a block
        _slots("slots_step", 128, 128, "step", 16, 4096),
        # a batch of 2000 requests, prompts and continued ones, 300 000 new tokens
        _slots("slots_mixed", 2000, 300000, "mixed", 16, 8192),
    ]


def _named(case, name):
    return dict(case, name=name) if name else case


def _patches(name, n, w, h, frames, patch, merge, group, dtype, filter, least=0, most=0):
    return _named({"kind": "patches", "n": n, "w_lo": w[0], "w_hi": w[1], "h_lo": h[0], "h_hi": h[1], "frames": frames, "patch": patch,
                   "merge": merge, "group": group, "dtype": dtype, "filter": filter, "least": least, "most": most}, name)


def _positions(name, n, capacity, content, merge):
    return _named({"kind": "positions", "n": n, "capacity": capacity, "content": content, "merge": merge}, name)


def _rotary(name, tokens, q_heads, k_heads, dim, sections, dtype, pairing, order, base, reach, store=False, slots=0, inverse=False,
            fused=False, ladder="shared"):
    return _named({"kind": "rotary", "tokens": tokens, "q_heads": q_heads, "k_heads": k_heads, "dim": dim, "st": sections[0],
                   "sh": sections[1], "sw": sections[2], "dtype": dtype, "pairing": pairing, "order": order, "base": base, "reach": reach,
                   "store": store, "slots": slots, "inverse": inverse, "fused": fused, "ladder": ladder}, name)


def _slots(name, n, capacity, content, block, width):
    return _named({"kind": "slots", "n": n, "capacity": capacity, "content": content, "block": block, "width": width}, name)


# ---- drawn cases ---------------------------------------------------------------------------------


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.random()
    if what < 0.35:
        w = _log(rng, 40, 1920)
        h = max(30, min(1088, int(w * rng.uniform(0.5, 1.5))))
        patch, merge, group = rng.choice((7, 8, 14, 14, 16, 16)), rng.choice((1, 2, 2, 3)), rng.choice((1, 1, 2))
        clip = rng.random() < 0.35
        most = max(1, min(96, 24000000 // (w * h)))
        n, frames = (1, _log(rng, 2, max(2, min(48, most)))) if clip else (_log(rng, 1, most), 1)
        ws, hs = ((max(30, int(w * 0.6)), w), (max(30, int(h * 0.6)), h)) if rng.random() < 0.5 else ((w, w), (h, h))
        cap = int(w * h * rng.uniform(0.1, 0.9)) if rng.random() < 0.5 else 0
        return _patches(None, n, ws, hs, frames, patch, merge, group, rng.choice(("bf16", "bf16", "f16", "f32")),
                        rng.choice(("antialias", "antialias", "bilinear")), least=0 if cap else rng.choice((0, 56 * 56)), most=cap)
    if what < 0.5:
        if rng.random() < 0.3:
            n = _log(rng, 1, 512)
            return _positions(None, n, n + rng.randint(0, 40), "step", 1)
        return _positions(None, _log(rng, 1, 512), _log(rng, 500, 400000), "mixed", rng.choice((1, 1, 2)))
    if what < 0.85:
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 256))
        pairs = rng.choice((dim // 2, dim // 2, dim // 4))
        h = rng.randint(0, pairs // 3)
        w = rng.randint(max(0, h - 1), h)
        sections = (pairs - h - w, h, w)
        kh = rng.choice((1, 2, 4, 8))
        qh = kh * rng.choice((1, 2, 4, 7, 8))
        while (qh + 2 * kh) * dim > 8192:
            qh -= kh
        qh = max(qh, kh)
        store = rng.random() < 0.4
        most = 40000000 // (qh + 2 * kh) // dim // (SIZES[dtype] // 2)
        tokens = _log(rng, 1, most)
        inverse = not store and rng.random() < 0.4
        return _rotary(None, tokens, qh, kh, dim, sections, dtype, rng.choice(("halves", "halves", "adjacent")),
                       rng.choice(("blocks", "interleaved")), rng.choice((10000.0, 500000.0, 1000000.0)), _log(rng, 100, 1000000),
                       store=store, slots=(tokens + tokens // 4 + 64) // 16 * 16 if store else 0, inverse=inverse,
                       fused=not store and rng.random() < 0.4, ladder=rng.choice(("shared", "axis")))
    if rng.random() < 0.4:
        n = _log(rng, 1, 1024)
        return _slots(None, n, n + rng.randint(0, 64), "step", rng.choice((8, 16, 32, 64)), 4096)
    return _slots(None, _log(rng, 1, 4096), _log(rng, 1000, 300000), "mixed", rng.choice((8, 16, 32, 64)), 8192)


# ---- inputs ----------------------------------------------------------------------------------------


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _sizes(case):
    """Width and height of every clip (they belong to the case, so that the outputs of every seed have one shape)."""
    rnd = np.random.default_rng(case["n"] * 7919 + case["w_hi"])
    return [(int(rnd.integers(case["w_lo"], case["w_hi"] + 1)), int(rnd.integers(case["h_lo"], case["h_hi"] + 1))) for _ in range(case["n"])]


def _target(case, w, h):
    """Size that an image of w x h is resized to."""
    u = case["patch"] * case["merge"]
    kw, kh = max(1, (2 * w + u) // (2 * u)), max(1, (2 * h + u) // (2 * u))
    pixels = kw * kh * u * u
    if case["most"] and pixels > case["most"]:
        kw = max(1, math.isqrt(w * case["most"] // (h * u * u)))
        kh = max(1, math.isqrt(h * case["most"] // (w * u * u)))
    elif pixels < case["least"]:
        def up(a, b):  # smallest k with k * k * b >= a
            k = math.isqrt(a // b)
            return k if k * k * b >= a else k + 1
        kw, kh = up(w * case["least"], h * u * u), up(h * case["least"], w * u * u)
    return kw * u, kh * u


def _rows(case):
    per, total = [], 0
    for w, h in _sizes(case):
        ow, oh = _target(case, w, h)
        t = -(-case["frames"] // case["group"])
        per.append((t, oh // case["patch"], ow // case["patch"]))
        total += t * (oh // case["patch"]) * (ow // case["patch"])
    return per, total


def _prepare_patches(case, seed):
    """Clips of smooth colour, edges and noise, with padded rows, one behind the other in one buffer."""
    gen = _generator(seed)
    offsets, pitches, parts, at = [], [], [], 0
    for w, h in _sizes(case):
        pitch = w * 3 + 5 if w % 2 else w * 3
        low = torch.rand((case["frames"], 3, 9, 9), generator=gen, device="cuda") * 255.0
        img = torch.nn.functional.interpolate(low, size=(h, w), mode="nearest")
        ramp = torch.linspace(-40.0, 40.0, w, device="cuda")[None, None, None, :]
        img = img + ramp + 8.0 * torch.randn(img.shape, generator=gen, device="cuda")
        img = img.round_().clamp_(0, 255).to(torch.uint8).permute(0, 2, 3, 1)
        rows = torch.zeros((case["frames"], h, pitch), dtype=torch.uint8, device="cuda")
        rows[:, :, :w * 3] = img.reshape(case["frames"], h, w * 3)
        offsets.append(at)
        pitches.append(pitch)
        parts.append(rows.reshape(-1))
        at += rows.numel()
    per, total = _rows(case)
    state = {"rgb": torch.cat(parts), "offsets": offsets, "pitches": pitches, "sizes": _sizes(case), "grids": per, "total": total,
             "rows": torch.zeros((total, 3 * case["group"] * case["patch"] ** 2), dtype=TYPES[case["dtype"]], device="cuda")}
    if own:
        import paper_2411_19114_amd as prep
        state["params"] = prep.make_patch_params(case["patch"], case["merge"], case["group"], case["dtype"], MEAN, STD,
                                                 prep.FILTER_ANTIALIAS if case["filter"] == "antialias" else prep.FILTER_BILINEAR,
                                                 min_pixels=case["least"], max_pixels=case["most"])
        state["widths"], state["heights"] = [s[0] for s in state["sizes"]], [s[1] for s in state["sizes"]]
        state["frames"] = [case["frames"]] * case["n"]
        state["strides"] = [h * p for (_, h), p in zip(state["sizes"], pitches)]
    return state


def _segment_lists(case, seed):
    """Host lists: segments of all sequences, and where each sequence's begin; at most `capacity` tokens in all."""
    rnd = np.random.default_rng(seed)
    segments, starts, left = [], [0], case["capacity"]
    for i in range(case["n"]):
        if case["content"] == "step":
            mine = [(1, 0, 0, 0)]
        else:
            mine = []
            budget = max(1, int(2 * rnd.random() * left / (case["n"] - i)))
            while budget > 0:
                text = int(min(budget, 1 + rnd.geometric(1 / 120.0)))
                mine.append((text, 0, 0, 0))
                budget -= text
                t = 1 if rnd.random() < 0.8 else int(rnd.integers(2, 13))
                h, w = int(rnd.integers(3, 37)), int(rnd.integers(3, 37))
                if t * h * w <= budget:
                    mine.append((t, h, w, int(rnd.integers(1, 5)) if t > 1 else 1))
                    budget -= t * h * w
        for s in mine:
            count = s[0] * max(s[1], 1) * max(s[2], 1)
            if count > left:
                s, count = (left, 0, 0, 0), left
            segments.append(s)
            left -= count
        starts.append(len(segments))
    first = rnd.integers(0, 30000, case["n"]) if case["content"] == "step" else np.zeros(case["n"])
    return segments, starts, first.astype(np.int32)


def _prepare_positions(case, seed):
    segments, starts, first = _segment_lists(case, seed)
    room = 4 * case["n"] + case["capacity"] // 4  # what such a program has room for
    padded = np.zeros((max(room, len(segments)), 4), dtype=np.int32)
    padded[:len(segments)] = segments
    state = {"segments": torch.from_numpy(padded[:len(segments)].copy()).cuda(), "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
             "first": torch.from_numpy(first).cuda(),
             "positions": torch.zeros((3, case["capacity"]), dtype=torch.int32, device="cuda"),
             "token_starts": torch.zeros(case["n"] + 1, dtype=torch.int32, device="cuda"),
             "next": torch.zeros(case["n"], dtype=torch.int32, device="cuda")}
    if own:
        import paper_2411_19114_amd as prep
        state["workspace"] = torch.zeros(prep.token_positions_workspace(len(segments)), dtype=torch.uint8, device="cuda")
    return state


def _axes(case):
    """Axis of every pair, and its place among the pairs of that axis."""
    st, sh, sw = case["st"], case["sh"], case["sw"]
    if case["order"] == "blocks":
        axes = [0] * st + [1] * sh + [2] * sw
    else:
        axes = [1 if i % 3 == 1 and i < 3 * sh else 2 if i % 3 == 2 and i < 3 * sw else 0 for i in range(st + sh + sw)]
    seen, place = [0, 0, 0], []
    for a in axes:
        place.append(seen[a])
        seen[a] += 1
    return axes, place


def _frequencies(case):
    """Radians a position for every pair, float64."""
    axes, place = _axes(case)
    n = (case["st"], case["sh"], case["sw"])
    if case["ladder"] == "axis":
        return np.array([case["base"] ** (-place[i] / n[a]) for i, a in enumerate(axes)])
    return np.array([case["base"] ** (-i / len(axes)) for i in range(len(axes))])


def _prepare_rotary(case, seed):
    gen = _generator(seed)
    n, qh, kh, d, dt = case["tokens"], case["q_heads"], case["k_heads"], case["dim"], TYPES[case["dtype"]]

    def random(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)

    heads = qh + 2 * kh
    if case["fused"] or case["store"]:  # views of one projection's output
        qkv = random(n, heads, d)
        q, k, v = qkv[:, :qh], qkv[:, qh:qh + kh], qkv[:, qh + kh:]
    else:
        q, k, v = random(n, qh, d), random(n, kh, d), None
    state = {"q": q, "k": k, "v": v, "q_out": torch.zeros((n, qh, d), dtype=dt, device="cuda"),
             "positions": torch.randint(0, case["reach"], (3, n), generator=gen, device="cuda", dtype=torch.int32)}
    if case["store"]:
        blocks = case["slots"] // 16
        for name in ("k_cache", "v_cache"):  # one block more than the pool, for rows that have no slot in the plain form
            state[name] = torch.zeros((blocks + 1, 16, kh, d), dtype=dt, device="cuda")
            state[name][:blocks] = random(blocks, 16, kh, d)
        slots = torch.randperm(blocks * 16, generator=gen, device="cuda")[:n].to(torch.int64)
        slots[torch.rand(n, generator=gen, device="cuda") < 0.02] = -1
        state["slots"] = slots
    else:
        state["k_out"] = torch.zeros((n, kh, d), dtype=dt, device="cuda")
    axes, _ = _axes(case)
    if own:
        import paper_2411_19114_amd as prep
        state["rotary"] = prep.Rotary(d, (case["st"], case["sh"], case["sw"]), case["base"], case["dtype"],
                                      pairing=prep.PAIR_HALVES if case["pairing"] == "halves" else prep.PAIR_ADJACENT,
                                      order=prep.SECTIONS_BLOCKS if case["order"] == "blocks" else prep.SECTIONS_INTERLEAVED,
                                      per_axis=case["ladder"] == "axis")
    else:
        state["axes"] = torch.tensor(axes, device="cuda")
        state["frequencies"] = torch.from_numpy(_frequencies(case)).cuda()
    return state


def _prepare_slots(case, seed):
    rnd = np.random.default_rng(seed)
    n, b = case["n"], case["block"]
    if case["content"] == "step":
        cached, fresh = rnd.integers(0, 3000, n), np.ones(n, dtype=np.int64)
    else:
        cached = np.where(rnd.random(n) < 0.5, 0, rnd.integers(0, 4000, n))
        fresh = np.where(rnd.random(n) < 0.3, 1, rnd.integers(0, max(2, 2 * case["capacity"] // n), n))
        fresh = np.minimum(fresh, 20000)
    end = np.minimum(np.cumsum(fresh), case["capacity"])
    fresh = np.diff(end, prepend=0)
    had, want = -(-cached // b), -(-(cached + fresh) // b)
    n_blocks = int(want.sum()) + 64
    order = rnd.permutation(n_blocks).astype(np.int32)
    table = np.zeros((n + 1, case["width"]), dtype=np.int32)  # a row behind the requests' for the plain form
    at = 0
    for i in range(n):
        table[i, :had[i]] = order[at:at + had[i]]
        at += int(had[i])
    free = np.zeros(n_blocks, dtype=np.int32)  # the stack has room for every block of the cache
    free[:n_blocks - at] = order[at:]
    state = {"cached": cached.astype(np.int32), "fresh": fresh.astype(np.int32), "free": free,
             "free_count": np.array([n_blocks - at], dtype=np.int32), "table": table}
    state = {k: torch.from_numpy(v).cuda() for k, v in state.items()}
    state.update(n_blocks=n_blocks, slots=torch.zeros(case["capacity"], dtype=torch.int64, device="cuda"),
                 token_starts=torch.zeros(n + 1, dtype=torch.int32, device="cuda"), lengths=torch.zeros(n, dtype=torch.int32, device="cuda"),
                 status=torch.zeros(n, dtype=torch.int32, device="cuda"), free_left=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2411_19114_amd as prep
        state["workspace"] = torch.zeros(prep.block_slots_workspace(n), dtype=torch.uint8, device="cuda")
    return state


def prepare(case, seed):
    state = {"patches": _prepare_patches, "positions": _prepare_positions, "rotary": _prepare_rotary, "slots": _prepare_slots}[case["kind"]](case, seed)
    state["case"] = case
    return state


# ---- one pass ----------------------------------------------------------------------------------------


def run(state):
    return {"patches": _run_patches, "positions": _run_positions, "rotary": _run_rotary, "slots": _run_slots}[state["case"]["kind"]](state)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _taps(size, out, filter):
    """Source samples and weights of every output sample of an axis: [out, taps] each (64 bits: borders of windows)."""
    c = (torch.arange(out, device="cuda", dtype=torch.float64) + 0.5) * size / out - 0.5
    s = size / out if filter == "antialias" else 1.0
    if s > 1.0:
        reach = int(math.floor(2 * s)) + 2
        j = torch.floor(c - s)[:, None] + torch.arange(1, reach + 1, device="cuda", dtype=torch.float64)
        weight = (1.0 - (j - c[:, None]).abs() / s).clamp_(min=0.0) * (j >= 0) * (j < size)
        weight = weight / weight.sum(1, keepdim=True)
    else:
        j = torch.floor(c)[:, None] + torch.arange(2, device="cuda", dtype=torch.float64)
        weight = (1.0 - (j - c[:, None]).abs())
    return j.clamp_(0, size - 1).to(torch.int64), weight.float()


def _run_patches(state):
    case = state["case"]
    if own:
        import paper_2411_19114_amd as prep
        prep.patch_rows(0, state["rgb"].data_ptr(), state["offsets"], state["widths"], state["heights"], state["pitches"], state["params"],
                        state["rows"].data_ptr(), state["total"], frames=state["frames"], frame_strides=state["strides"], stream=_stream())
        return state["rows"]
    p, m, g, f = case["patch"], case["merge"], case["group"], case["frames"]
    mean = torch.tensor(MEAN, device="cuda")
    std = torch.tensor(STD, device="cuda")
    at = 0
    for (w, h), offset, pitch, (t, gh, gw) in zip(state["sizes"], state["offsets"], state["pitches"], state["grids"]):
        img = state["rgb"][offset:offset + f * h * pitch].reshape(f, h, pitch)[:, :, :3 * w].reshape(f, h, w, 3)
        jy, wy = _taps(h, gh * p, case["filter"])
        jx, wx = _taps(w, gw * p, case["filter"])
        tall = torch.zeros((f, gh * p, w, 3), device="cuda")
        for k in range(jy.shape[1]):
            tall += img[:, jy[:, k]].float() * wy[:, k][None, :, None, None]
        out = torch.zeros((f, gh * p, gw * p, 3), device="cuda")
        for k in range(jx.shape[1]):
            out += tall[:, :, jx[:, k]] * wx[:, k][None, None, :, None]
        out = (out / 255.0 - mean) / std
        if f < t * g:
            out = torch.cat([out] + [out[-1:]] * (t * g - f))
        rows = out.reshape(t, g, gh // m, m, p, gw // m, m, p, 3).permute(0, 2, 5, 3, 6, 8, 1, 4, 7)
        state["rows"][at:at + t * gh * gw] = rows.reshape(t * gh * gw, -1).to(TYPES[case["dtype"]])
        at += t * gh * gw
    return state["rows"]


def _run_positions(state):
    case = state["case"]
    n, capacity = case["n"], case["capacity"]
    segments, starts = state["segments"], state["starts"]
    if own:
        import paper_2411_19114_amd as prep
        prep.token_positions(segments.data_ptr(), segments.shape[0], starts.data_ptr(), n, state["first"].data_ptr(), case["merge"],
                             state["positions"].data_ptr(), capacity, state["token_starts"].data_ptr(), state["next"].data_ptr(),
                             state["workspace"].data_ptr(), state["workspace"].numel(), stream=_stream())
        return state["positions"], state["token_starts"], state["next"]
    t, h, w, step = (segments[:, i].to(torch.int64) for i in range(4))
    text = h == 0
    count = torch.where(text, t, t * h * w)
    advance = torch.where(text, t, torch.maximum(torch.maximum((t - 1) * step, h - 1), w - 1) + 1)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    tokens = torch.cat([zero, torch.cumsum(count, 0)])
    moved = torch.cat([zero, torch.cumsum(advance, 0)])
    begin, end = starts[:-1].to(torch.int64), starts[1:].to(torch.int64)
    sequence = torch.searchsorted(end, torch.arange(segments.shape[0], device="cuda"), right=True)
    base = state["first"][sequence] + moved[:-1] - moved[begin][sequence]
    index = torch.arange(capacity, device="cuda")
    mine = torch.searchsorted(tokens[1:], index, right=True)
    real = mine < segments.shape[0]
    mine = mine.clamp(max=segments.shape[0] - 1)
    r = index - tokens[mine]
    hs, ws, m = h[mine].clamp(min=1), w[mine].clamp(min=1), case["merge"]
    frame, r2 = r // (hs * ws), r % (hs * ws)
    band = r2 // (m * ws)
    r3 = r2 - band * m * ws
    tall = torch.minimum(hs - band * m, torch.full_like(hs, m))
    window = r3 // (tall * m)
    r4 = r3 - window * tall * m
    wide = torch.minimum(ws - window * m, torch.full_like(ws, m))
    y, x = band * m + r4 // wide, window * m + r4 % wide
    is_text = text[mine]
    p = base[mine]
    out = torch.stack([torch.where(is_text, p + r, p + frame * step[mine]), torch.where(is_text, p + r, p + y), torch.where(is_text, p + r, p + x)])
    state["positions"].copy_(torch.where(real, out, torch.zeros_like(out)))
    state["token_starts"].copy_(tokens[starts.to(torch.int64)])
    state["next"].copy_(state["first"] + moved[end] - moved[begin])
    return state["positions"], state["token_starts"], state["next"]


def _rotate(x, cos, sin, pairing, inverse):
    """x [tokens, heads, dim] by the angles of [tokens, pairs]; values behind the rotated ones stay."""
    pairs = cos.shape[1]
    x = x.float()
    c, s = cos[:, None], -sin[:, None] if inverse else sin[:, None]
    out = x.clone()
    if pairing == "halves":
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        out[..., :pairs], out[..., pairs:2 * pairs] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        out[..., 0:2 * pairs:2], out[..., 1:2 * pairs:2] = a * c - b * s, a * s + b * c
    return out


def _run_rotary(state):
    case = state["case"]
    n, kh, d = case["tokens"], case["k_heads"], case["dim"]
    q, k, v = state["q"], state["k"], state["v"]
    if own:
        def view(x):
            return x.data_ptr(), x.stride(0), x.stride(1)
        if case["store"]:
            cache = state["k_cache"]
            state["rotary"].apply(n, state["positions"].data_ptr(), n, q=view(q), q_out=view(state["q_out"]), q_heads=case["q_heads"],
                                  k=view(k), k_heads=kh, v=view(v), k_cache=cache.data_ptr(), v_cache=state["v_cache"].data_ptr(),
                                  n_blocks=cache.shape[0] - 1, block_size=16, block_stride=cache.stride(0), slot_stride=cache.stride(1),
                                  cache_head_stride=cache.stride(2), slots=state["slots"].data_ptr(), stream=_stream())
            return state["q_out"], state["k_cache"][:-1], state["v_cache"][:-1]
        state["rotary"].apply(n, state["positions"].data_ptr(), n, q=view(q), q_out=view(state["q_out"]), q_heads=case["q_heads"], k=view(k),
                              k_out=view(state["k_out"]), k_heads=kh, inverse=case["inverse"], stream=_stream())
        return state["q_out"], state["k_out"]
    angle = state["positions"][state["axes"]].T.double() * state["frequencies"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    state["q_out"].copy_(_rotate(q, cos, sin, case["pairing"], case["inverse"]))
    turned = _rotate(k, cos, sin, case["pairing"], case["inverse"])
    if not case["store"]:
        state["k_out"].copy_(turned)
        return state["q_out"], state["k_out"]
    at = torch.where(state["slots"] < 0, case["slots"], state["slots"])
    state["k_cache"].view(-1, kh, d)[at] = turned.to(k.dtype)
    state["v_cache"].view(-1, kh, d)[at] = v
    return state["q_out"], state["k_cache"][:-1], state["v_cache"][:-1]


def _run_slots(state):
    case = state["case"]
    n, b, capacity, table = case["n"], case["block"], case["capacity"], state["table"]
    if own:
        import paper_2411_19114_amd as prep
        prep.block_slots(n, b, state["n_blocks"], state["cached"].data_ptr(), state["fresh"].data_ptr(), state["free"].data_ptr(),
                         state["free"].numel(), state["free_count"].data_ptr(), table.data_ptr(), table.stride(0), case["width"],
                         state["slots"].data_ptr(), capacity, state["token_starts"].data_ptr(), state["lengths"].data_ptr(),
                         state["status"].data_ptr(), state["free_left"].data_ptr(), state["workspace"].data_ptr(),
                         state["workspace"].numel(), stream=_stream())
    else:
        cached, fresh = state["cached"].to(torch.int64), state["fresh"].to(torch.int64)
        had, want = (cached + b - 1) // b, (cached + fresh + b - 1) // b
        zero = torch.zeros(1, dtype=torch.int64, device="cuda")
        starts = torch.cat([zero, torch.cumsum(fresh, 0)])
        fits = (want <= case["width"]) & (starts[1:] <= capacity)
        need = torch.where(fits, want - had, torch.zeros_like(want))
        taken = torch.cumsum(need, 0)
        granted = fits & (taken <= state["free_count"])
        index = torch.arange(capacity, device="cuda")
        mine = torch.searchsorted(starts[1:], index, right=True)
        real = mine < n
        mine = mine.clamp(max=n - 1)
        real = real & granted[mine]
        place = cached[mine] + index - starts[mine]
        block = place // b
        fresh_block = block >= had[mine]
        k = (taken - need)[mine] + block - had[mine]
        popped = state["free"][(state["free_count"] - 1 - k).clamp(0, state["free"].numel() - 1)]
        kept = table[mine, block.clamp(0, case["width"] - 1)]
        block_id = torch.where(fresh_block, popped, kept).to(torch.int64)
        state["slots"].copy_(torch.where(real, block_id * b + place % b, torch.full_like(place, -1)))
        # every token of a new block puts it into the table, the others write into the row behind
        row = torch.where(real & fresh_block, mine, n)
        table[row, block.clamp(0, case["width"] - 1)] = popped
        state["token_starts"].copy_(starts)
        state["lengths"].copy_(torch.where(granted, cached + fresh, cached))
        state["status"].copy_(torch.where(granted, 0, -2))
        state["free_left"].copy_(state["free_count"] - torch.where(granted, taken, torch.zeros_like(taken)).max())
    return state["slots"], table[:n], state["token_starts"], state["lengths"], state["status"], state["free_left"]


# ---- the work of a pass, and what it should have given ---------------------------------------------------


def work(case):
    if case["kind"] == "patches":
        _, rows = _rows(case)
        pixels = values = flops = 0
        for w, h in _sizes(case):
            ow, oh = _target(case, w, h)
            sx, sy = (max(1.0, w / ow), max(1.0, h / oh)) if case["filter"] == "antialias" else (1.0, 1.0)
            pixels += case["frames"] * w * h
            values += case["frames"] * 3 * ow * oh
            flops += case["frames"] * 3 * oh * (4.0 * sy * w + 4.0 * sx * ow)
        return {"bytes": 3 * pixels + rows * 3 * case["group"] * case["patch"] ** 2 * SIZES[case["dtype"]], "flops": flops + 2 * values}
    if case["kind"] == "positions":
        return {"bytes": 12 * case["capacity"] + 28 * case["n"], "flops": 12 * case["capacity"]}
    if case["kind"] == "rotary":
        heads = case["q_heads"] + case["k_heads"] * (2 if case["store"] else 1)
        pairs = case["st"] + case["sh"] + case["sw"]
        return {"bytes": case["tokens"] * (2 * heads * case["dim"] * SIZES[case["dtype"]] + 12 + (8 if case["store"] else 0)),
                "flops": case["tokens"] * pairs * (6 * (case["q_heads"] + case["k_heads"]) + 24)}
    return {"bytes": 8 * case["capacity"] + 20 * case["n"] + 8 * case["capacity"] // case["block"], "flops": 8 * case["capacity"]}


def exact(case, seed):
    return {"patches": _exact_patches, "positions": _exact_positions, "rotary": _exact_rotary, "slots": _exact_slots}[case["kind"]](case, seed)


def _weights(size, out, antialias):
    """Dense [out, size] weights of one axis in 64 bits."""
    m = np.zeros((out, size))
    scale = size / out
    for i in range(out):
        centre = (i + 0.5) * scale
        if antialias and scale > 1.0:
            lo, hi = max(0, math.floor(centre - scale) - 1), min(size, math.ceil(centre + scale) + 1)
            j = np.arange(lo, hi)
            v = np.maximum(0.0, 1.0 - np.abs(j + 0.5 - centre) / scale)
            m[i, lo:hi] = v / v.sum()
        else:
            a = math.floor(centre - 0.5)
            part = centre - 0.5 - a
            m[i, min(max(a, 0), size - 1)] += 1.0 - part
            m[i, min(max(a + 1, 0), size - 1)] += part
    return torch.from_numpy(m).cuda()


def _exact_patches(case, seed):
    state = _prepare_patches(case, seed)
    p, m, g, f = case["patch"], case["merge"], case["group"], case["frames"]
    out = torch.empty((state["total"], 3 * g * p * p), dtype=torch.float64, device="cuda")
    at = 0
    for (w, h), offset, pitch in zip(state["sizes"], state["offsets"], state["pitches"]):
        ow, oh = _target(case, w, h)
        wy, wx = _weights(h, oh, case["filter"] == "antialias"), _weights(w, ow, case["filter"] == "antialias")
        frames = []
        for i in range(f):
            img = state["rgb"][offset + i * h * pitch:offset + (i + 1) * h * pitch].reshape(h, pitch)[:, :3 * w].reshape(h, w, 3).double()
            planes = []
            for c in range(3):
                v = wy @ img[:, :, c].contiguous() @ wx.T.contiguous()
                planes.append((v / 255.0 - MEAN[c]) / STD[c])
            frames.append(torch.stack(planes))
        gh, gw = oh // p, ow // p
        order = [(y * m + a, x * m + b) for y in range(gh // m) for x in range(gw // m) for a in range(m) for b in range(m)]
        order = torch.tensor([a * gw + b for a, b in order], device="cuda")
        for t in range(-(-f // g)):
            group = torch.stack([frames[min(t * g + i, f - 1)] for i in range(g)], 1)  # [3, g, oh, ow]
            cut = group.unfold(2, p, p).unfold(3, p, p)  # [3, g, gh, gw, p, p]
            cut = cut.permute(2, 3, 0, 1, 4, 5).reshape(gh * gw, -1)
            out[at:at + gh * gw] = cut[order]
            at += gh * gw
    return out


def _exact_positions(case, seed):
    segments, starts, first = _segment_lists(case, seed)
    positions = np.zeros((3, case["capacity"]), dtype=np.int64)
    token_starts, nexts, at, m = [0], [], 0, case["merge"]
    for i in range(case["n"]):
        p = int(first[i])
        for t, h, w, step in segments[starts[i]:starts[i + 1]]:
            if h == 0:
                positions[:, at:at + t] = p + np.arange(t)
                at += t
                p += t
                continue
            y, x = np.mgrid[0:h, 0:w]
            key = np.lexsort((x.ravel(), y.ravel(), x.ravel() // m, y.ravel() // m))  # windows in raster order, then inside
            for a in range(t):
                positions[0, at:at + h * w] = p + a * step
                positions[1, at:at + h * w] = p + y.ravel()[key]
                positions[2, at:at + h * w] = p + x.ravel()[key]
                at += h * w
            p += max((t - 1) * step, h - 1, w - 1) + 1
        token_starts.append(at)
        nexts.append(p)
    return (torch.from_numpy(positions.astype(np.int32)), torch.tensor(token_starts, dtype=torch.int32), torch.tensor(nexts, dtype=torch.int32))


def _exact_rotary(case, seed):
    state = _prepare_rotary(case, seed)
    axes, _ = _axes(case)
    f = _frequencies(case)
    n = case["tokens"]

    def turn(x):
        out = x.double().clone()
        pairs = len(axes)
        for i in range(pairs):
            a, b = (i, i + pairs) if case["pairing"] == "halves" else (2 * i, 2 * i + 1)
            angle = state["positions"][axes[i]].double() * float(f[i])
            z = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)[:, None]
            z = z * torch.complex(x[..., a].double(), x[..., b].double())
            out[..., a], out[..., b] = z.real, z.imag
        return out

    q, k = turn(state["q"]), turn(state["k"])
    if not case["store"]:
        return q, k
    caches = [state[name][:-1].double().reshape(-1, case["k_heads"], case["dim"]) for name in ("k_cache", "v_cache")]
    kept = torch.nonzero(state["slots"] >= 0).flatten()
    caches[0][state["slots"][kept]] = k[kept]
    caches[1][state["slots"][kept]] = state["v"][kept].double()
    shape = (case["slots"] // 16, 16, case["k_heads"], case["dim"])
    assert n == q.shape[0]
    return q, caches[0].reshape(shape), caches[1].reshape(shape)


def _exact_slots(case, seed):
    state = {k: v.cpu().numpy() if torch.is_tensor(v) else v for k, v in _prepare_slots(case, seed).items()}
    b, table, stack = case["block"], state["table"].copy(), list(state["free"][:int(state["free_count"][0])])
    slots, starts, lengths, status = [], [0], [], []
    for i in range(case["n"]):
        c, f = int(state["cached"][i]), int(state["fresh"][i])
        had, want = -(-c // b), -(-(c + f) // b)
        for j in range(had, want):
            table[i, j] = stack.pop()
        place = np.arange(c, c + f)
        slots.append(table[i, place // b].astype(np.int64) * b + place % b)
        starts.append(starts[-1] + f)
        lengths.append(c + f)
        status.append(0)
    slots.append(np.full(case["capacity"] - starts[-1], -1, dtype=np.int64))
    return (torch.from_numpy(np.concatenate(slots)), torch.from_numpy(table[:case["n"]].copy()), torch.tensor(starts, dtype=torch.int32),
            torch.tensor(lengths, dtype=torch.int32), torch.tensor(status, dtype=torch.int32), torch.tensor([len(stack)], dtype=torch.int32))
