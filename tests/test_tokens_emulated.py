"""The operators for packed batches of tokens without a GPU: their sources compiled by g++ against the CPU stand-in
for HIP (AddressSanitizer and UBSan on), called through the binding, against the oracle.  The same checks run on the GPU
in test_gpu_tokens.py."""
import os
import subprocess
import sys

import pytest

import emul
import token_cases as cases

LIBRARY = os.path.join(emul.EMU, "prep_emul_lib")
SOURCES = emul.KERNELS + [k for k in ("patches.hip", "packing.hip", "rotary.hip") if k not in emul.KERNELS]


def build():
    srcs = [os.path.join(emul.CSRC, k) for k in SOURCES] + [os.path.join(emul.EMU, "emul_runtime.cpp")]
    deps = srcs + [os.path.join(emul.CSRC, x) for x in ("kernels.h", "parser.h", "prep_internal.h", "tokens.h", "matrix.h")] + \
        [os.path.join(emul.ROOT, "include", "prep.h"), os.path.join(emul.EMU, "more_hip.h")] + [os.path.join(emul.EMU, "hip", x) for x in os.listdir(os.path.join(emul.EMU, "hip"))]
    if os.path.exists(LIBRARY) and os.path.getmtime(LIBRARY) >= max(os.path.getmtime(d) for d in deps):
        return
    subprocess.run(["g++", "-std=c++20", "-O1", "-g", "-pthread", "-fPIC", "-shared", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=undefined", "-I", emul.EMU, "-include", os.path.join(emul.EMU, "more_hip.h"), "-x", "c++"] + srcs + ["-o", LIBRARY], check=True)


def run(*checks):
    build()
    asan = subprocess.run(["g++", "-print-file-name=libasan.so"], capture_output=True, text=True, check=True).stdout.strip()
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0")
    r = subprocess.run([sys.executable, os.path.join(emul.ROOT, "tests", "tokens_on_cpu.py"), LIBRARY, *checks], capture_output=True, text=True,
                       timeout=900, env=env)
    assert r.returncode == 0 and r.stdout.endswith("all passed\n"), r.stdout[-500:] + r.stderr[-4000:]


def test_argument_blocks_are_packed_as_the_sources_declare_them():
    import paper_2411_19114_amd.binding as binding
    for packed, source in ((binding._BLOCK_ARGS, "packing.hip"), (binding._ROTARY_ARGS, "rotary.hip")):
        assert f"_args) == {packed.size}," in open(os.path.join(emul.CSRC, source)).read()


def _some(names, k, of):
    return [n for i, n in enumerate(names) if i % of == k]


@pytest.mark.parametrize("k", range(4))
def test_patch_rows(k):
    run(*(f"check_patches:{n}" for n in _some(cases.PATCHES, k, 4)))


def test_places():
    run(*(f"check_positions:{n}" for n in cases.POSITIONS))


def test_slots():
    run(*(f"check_slots:{n}" for n in cases.SLOTS), "check_bad_blocks")


@pytest.mark.parametrize("k", range(3))
def test_rotary(k):
    run(*(f"check_rotary:{n}" for n in _some(cases.ROTARY, k, 3)))


def test_rotary_gradient():
    run("check_rotary_gradient:False", "check_rotary_gradient:True")


def test_refusals():
    run("check_patch_refusals", "check_packing_refusals", "check_rotary_refusals")


def test_more_tokens_than_64_bits_count():
    run("check_more_tokens_than_64_bits_count")


def test_slow_pairs():
    run("check_slow_pairs:False", "check_slow_pairs:True")


@pytest.mark.parametrize("name", cases.PATCHES_MORE)
def test_more_patch_rows(name):
    run(f"check_more_patches:{name}")


def test_given_frequencies():
    run("check_given_frequencies:False", "check_given_frequencies:True")


def test_segments_of_no_sequence():
    run("check_segments_of_no_sequence:False", "check_segments_of_no_sequence:True")
