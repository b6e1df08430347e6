"""The loss's two passes on the host: at many drawn sizes, every buffer of the
workspace lies within it and apart from the others, the kernels can fetch what they are
given, and every kernel that can be chosen is run by a GPU test."""
import math
import os
import random
import subprocess

import pytest
import torch

import test_gpu_tokens as gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def passes(tmp_path_factory):
    """f(lines): the products of each line's two passes."""
    exe = tmp_path_factory.mktemp("dispatch") / "tokens_dispatch"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-w", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROCM, "include"), "-I",
                    os.path.join(ROOT, "paper_2606_27153_amd", "csrc", "layers"),
                    os.path.join(ROOT, "tests", "tokens_dispatch.cpp"), "-o", str(exe)], check=True)

    def run(lines):
        out = subprocess.run([str(exe)], input="\n".join(lines), capture_output=True, text=True)
        assert out.returncode == 0, out.stdout[-300:] + out.stderr[-2000:]
        got = out.stdout.splitlines()
        assert len(got) == len(lines)
        bad = [(a, b) for a, b in zip(lines, got) if "FAILED" in b]
        assert not bad, bad[:3]
        return [line.split() for line in got]
    return run


def _line(dtype, transposed, rows, inner, vocab, off=0, reduction=2):
    return f"{int(dtype == torch.bfloat16)} {int(transposed)} {rows} {inner} {vocab} {off} {reduction}"


def _listed():
    both = [(d, t) for d in (torch.float32, torch.bfloat16) for t in (False, True)]
    out = [_line(d, t, *s) for s in gpu.LOSSES for d, t in both]
    return out + [_line(dtype, transposed, rows, inner, vocab) for rows, inner, vocab, transposed, dtype in gpu.LARGE]


def _drawn(n):
    rng = random.Random(3)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    lines = []
    for _ in range(n):
        inner = rng.choice((256, 1024, 2048, 4096)) if rng.random() < 0.5 else log(1, 8192)
        vocab = rng.choice((32000, 65536, 128000)) if rng.random() < 0.5 else log(1, 400000)
        lines.append(f"{rng.randrange(2)} {rng.randrange(2)} {log(1, 65536)} {inner} {vocab} "
                     f"{rng.choice((0, 0, 1, 3))} {rng.randrange(3)}")
    return lines


def test_buffers_lie_in_the_workspace_and_apart(passes):
    far = ["1 0 1048576 64 128000 0 2", "0 1 300000 4096 50001 1 1", "1 0 100 1048576 3000 0 2",
           "0 0 70 1048573 1000 0 0", "1 0 40000 256 16777216 0 2", "1 1 5 64 16777213 3 2", "0 0 0 16 40 0 2"]
    passes(_drawn(20000) + far + _listed())


def test_every_reachable_kernel_has_a_gpu_case(passes):
    covered = {w for words in passes(_listed()) for w in words}
    missing = {}
    lines = _drawn(20000)
    for line, words in zip(lines, passes(lines)):
        for w in words:
            if w not in covered:
                missing.setdefault(w, line)
    assert not missing, missing
    for w in ("strips/tile256/bf16/RT/0", "dz/tile256/bf16/RR/0", "weight/tile64/f32/TT/1", "dz/rows/bf16"):
        assert w in covered


def test_very_large_vocabularies_are_taken_in_fewer_rows_at_a_time(passes):
    """(The buffers in bounds and apart, as above, where rows and columns both come in pieces.)"""
    words = passes([f"{bf16} {t} {rows} 16 {vocab} {off} 2" for bf16 in (0, 1) for t in (0, 1)
                    for rows in (300, 5000, 40000) for vocab in (524288, 3000001, 1 << 24) for off in (0, 1)])
    assert all(w for w in words)


def test_last_pieces_of_few_rows_have_columns_enough(passes):
    """Columns that 32768 at a time would leave 1 to 7 of: the kernel of few rows reads 16
    bytes of them."""
    vocabs = [v for v in range(32768 * 127 + 1, 1 << 24, 32768) for v in (v, v + 2, v + 6)][::13]
    words = passes([f"{bf16} 0 {rows} 8 {v} 1 2" for bf16 in (0, 1) for rows in (1, 20) for v in vocabs])
    assert all(any(w.startswith("logits/skinny") for w in line) for line in words)


def test_weight_gradients_of_few_rows_by_size(passes):
    """The outer product where its streamed stores count, the tiles where the gradient is small."""
    cases = [  # rows, inner, vocab, transposed, dtype, outer product
        (1, 64, 1000, False, torch.bfloat16, True), (4, 256, 16384, True, torch.bfloat16, True),
        (8, 200, 10727, False, torch.float32, True), (8, 4096, 128000, False, torch.bfloat16, True),
        (8, 200, 10727, True, torch.bfloat16, True), (8, 200, 10727, False, torch.bfloat16, False),
        (8, 4096, 2000, True, torch.bfloat16, False), (6, 512, 32000, False, torch.bfloat16, True),
        (16, 200, 10727, True, torch.float32, True), (16, 256, 16384, False, torch.float32, False),
        (10, 200, 10727, True, torch.bfloat16, False), (16, 1024, 65536, True, torch.bfloat16, False),
        (16, 2048, 65536, True, torch.bfloat16, True), (9, 4096, 128000, False, torch.bfloat16, True),
        (32, 256, 32000, True, torch.float32, False), (20, 1408, 32000, False, torch.float32, True),
        (32, 1024, 32000, True, torch.float32, True), (16, 2048, 32000, True, torch.bfloat16, False),
        (17, 4096, 128000, False, torch.bfloat16, False), (33, 4096, 128000, False, torch.float32, False)]
    words = passes([_line(dtype, t, rows, inner, vocab) for rows, inner, vocab, t, dtype, _ in cases])
    for line, case in zip(words, cases):
        assert any(w.startswith("weight/outer") for w in line) == case[-1], (case, line)
        assert sum(w.startswith("weight") for w in line) == 1, line
