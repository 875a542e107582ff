"""The operators for packed batches of tokens on the GPU: calls whose sizes pass 32 bits, and what test_gpu_tokens.py leaves out."""
import numpy as np
import pytest

import paper_2411_19114_amd as prep
import token_cases as cases
from test_gpu_tokens import Backend
from test_token_limits import MOST, enlarging_weights, place_of_row

pytestmark = pytest.mark.gpu


def test_pictures_of_more_than_2_31_pixels():
    """Two stills of 2^31 pixels and some: rows on both sides of that pixel, at the seam of the two launches, and outside."""
    import torch
    w, patch, merge, side = 16, 16, 2, 46368
    params = prep.make_patch_params(patch, merge, 1, "bf16", cases.MEAN, cases.STD, prep.FILTER_ANTIALIAS, min_pixels=side * side)
    cols, area = side // patch, patch * patch
    rows = cols * cols
    assert 2 * rows * area > MOST
    pictures = cases.picture(np.random.default_rng(4), (2, w, w, 3))
    src = torch.from_numpy(pictures.reshape(-1)).cuda()
    out = torch.full((2 * rows + 2, 3 * area), -77.0, dtype=torch.bfloat16, device="cuda")
    print("2 stills of", side, "x", side, flush=True)
    starts = prep.patch_rows(0, src.data_ptr(), [0, w * w * 3], [w, w], [w, w], [3 * w] * 2, params, out.data_ptr() + 2 * 3 * area, 2 * rows,
                             stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert starts == [0, rows, 2 * rows]
    assert (out[0] == -77).all() and (out[-1] == -77).all()
    assert (out[1:-1] != -77).all(dim=1).all()  # (values lie between -2.2 and 2.7)
    weights = enlarging_weights(w, side)
    edge, seam = 2 ** 31 // area, MOST // 256
    for r in (0, 1, edge - 1, edge, edge + 1, rows - 1, rows, rows + edge - 1, seam - 1, seam, seam + 1, 2 * rows - 1):
        picture, row = divmod(r, rows)
        y, x = place_of_row(row, cols, merge)
        wy, wx = weights(range(y * patch, (y + 1) * patch)), weights(range(x * patch, (x + 1) * patch))
        v = np.stack([wy @ pictures[picture, ..., c].astype(np.float64) @ wx.T for c in range(3)])
        want = ((v / 255 - np.array(cases.MEAN)[:, None, None]) / np.array(cases.STD)[:, None, None]).ravel()
        cases.within(out[1 + r].cpu().double().numpy(), want, cases.patch_tolerance(w, w, side, side, True), "bf16")


def test_more_tokens_than_a_launch_has_work_items():
    """A pair a token, 2^27 tokens and some: two launches of rotary_pairs, against cos and sin in 64 bits."""
    import torch
    n = 8 * (MOST // 256) + 1003
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn((n, 2), device="cuda", generator=gen).to(torch.bfloat16)
    places = torch.randint(0, 100000, (n,), dtype=torch.int32, device="cuda", generator=gen)
    out = torch.full((n + 1, 2), 7.0, dtype=torch.bfloat16, device="cuda")
    rotary = prep.Rotary(2, (1, 0, 0), 1e4, "bf16")
    print(n, "tokens of a pair", flush=True)
    rotary.apply(n, places.data_ptr(), n, q=(x.data_ptr(), 2, 2), q_out=(out.data_ptr(), 2, 2), q_heads=1, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    rotary.close()
    assert (out[n:] == 7).all()
    step = 1 << 24
    for at in range(0, n, step):
        a, b = x[at:at + step].double().unbind(1)
        c, s = (f(places[at:at + step].double()) for f in (torch.cos, torch.sin))
        for got, want in zip(out[at:at + step].double()[:n - at].unbind(1), (a * c - b * s, a * s + b * c)):
            limit = (a.abs() + b.abs()) * (cases.TRIG + 2 * cases.ULP) * (1 + cases.HALF_STEP["bf16"]) + want.abs() * cases.HALF_STEP["bf16"] + cases.LEAST_STEP["bf16"]
            assert ((got - want).abs() <= limit).all(), at


def test_more_tokens_than_64_bits_count():
    cases.check_more_tokens_than_64_bits_count(Backend())


@pytest.mark.parametrize("adjacent", [False, True])
def test_slow_pairs(adjacent):
    cases.check_slow_pairs(Backend(), adjacent)


@pytest.mark.parametrize("name", cases.PATCHES_MORE | cases.PATCHES_MIXED)
def test_more_patch_rows(name):
    cases.check_more_patches(Backend(), name)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_given_frequencies(adjacent, dtype):
    cases.check_given_frequencies(Backend(), adjacent, dtype)


@pytest.mark.parametrize("many", [False, True])
def test_segments_of_no_sequence(many):
    cases.check_segments_of_no_sequence(Backend(), many)
