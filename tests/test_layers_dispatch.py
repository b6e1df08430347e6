"""Every kernel that the layer operators can choose is run by a GPU test: the
choice (kernel, operand layout, grouping, whether the sum is cut) of the listed
GPU cases is held against that of many drawn sizes.  Host only: the library's
entry points with launchers that note what they are asked to run."""
import math
import os
import random
import subprocess

import pytest
import torch

import layers_ref as R
import test_gpu_layers as small
import test_gpu_layers_dispatch as rest
import test_gpu_layers_large as large

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """f(lines): the launches of each line's two passes."""
    exe = tmp_path_factory.mktemp("dispatch") / "layers_dispatch"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-w", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROCM, "include"), "-I",
                    os.path.join(ROOT, "paper_2606_27153_amd", "csrc", "layers"),
                    os.path.join(ROOT, "tests", "layers_dispatch.cpp"), "-o", str(exe)], check=True)

    def run(lines):
        out = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True)
        assert out.returncode == 0 and "FAILED" not in out.stdout, out.stdout[-300:] + out.stderr[-2000:]
        got = [line.split() for line in out.stdout.splitlines()]
        assert len(got) == len(lines) and all(got)
        return got
    return run


def _linear(rows, inner, outer, dtype, act, transposed):
    return f"l {int(dtype == torch.bfloat16)} {int(transposed)} {rows} {inner} {outer} 0 {R.ACTS.index(act)}"


def _grouped(experts, rows, inner, outer, dtype, transposed):
    return f"g {int(dtype == torch.bfloat16)} {int(transposed)} {rows} {inner} {outer} {experts} 0"


def _params(test, name):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0].startswith(name))


def _listed():
    both = [(d, t) for d in (torch.float32, torch.bfloat16) for t in (False, True)]
    out = [_linear(*s, d, R.ACTS[sum(s) % 5], t) for s in small.SHAPES for d, t in both]
    out += [_linear(*c) for c in large.CASES + rest.LINEAR]
    for f in (large.test_grouped_large, large.test_grouped_few_rows_long_sums):
        out += [_grouped(*c) for c in _params(f, "experts")]
    out += [_grouped(*c) for c in rest.GROUPED]
    for counts, inner, outer in small.GROUPED:
        rows = sum(counts) + sum(counts) % 3 * 5 + sum(counts) % 4 * 9
        out += [_grouped(len(counts), rows, inner, outer, d, t) for d, t in both]
    return out


def test_every_reachable_kernel_has_a_gpu_case(launches):
    covered = {w for words in launches(_listed()) for w in words}
    rng = random.Random(1)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    widths = (256, 768, 1024, 1152, 1408, 2048, 3456, 4096, 4304, 5632, 14336)
    lines = []
    for _ in range(60000):
        op = rng.choice("lg")
        bf16, transposed = rng.randrange(2), rng.randrange(2)
        inner, outer = (rng.choice(widths), rng.choice(widths)) if rng.random() < 0.5 else (log(1, 16384), log(1, 16384))
        lines.append(f"{op} {bf16} {transposed} {log(1, 65536)} {inner} {outer} {log(1, 256) if op == 'g' else 0} "
                     f"{rng.randrange(5) if op == 'l' else 0}")
    missing = {}
    for line, words in zip(lines, launches(lines)):
        for w in words:
            if w not in covered:
                missing.setdefault(w, line)
    assert not missing, missing
    # the fp32 and bf16 tiles, whole and cut, are among them
    for w in ("tile128/f32/RT/plain/0", "tile128/f32/TT/plain/1", "tile256/bf16/RR/rows/1", "tile64/f32/TT/sum/0"):
        assert w in covered


def test_operands_are_copied_where_the_workspace_has_room(launches):
    """Odd sizes take the tile kernels too (the simple one is for callers that give no room)."""
    for words in launches(["l 1 0 1001 1003 1005 0 2", "l 0 1 1001 1003 1005 0 2", "g 1 0 1001 1003 1005 7 0"]):
        assert len(words) == 3 and not any("simple" in w for w in words)
