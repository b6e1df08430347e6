"""The layer library's C ABI without a GPU: exports, bindings, argument checks
(which come before any device call) and the kernels' register budget."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2606_27153_amd import _layers_lib as LL
from paper_2606_27153_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "muon_layers.h")
READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")


@pytest.fixture(scope="module")
def lay():
    return LL.load()


def test_every_declared_function_is_exported_and_bound(lay):
    txt = open(HEADER).read()
    names = sorted(set(re.findall(r"^MUON_API\s+[\w\s\*]+?\b(muon_\w+)\(", txt, flags=re.M)))
    assert names == sorted(LL.SIGNATURES)
    for n in names:
        assert hasattr(lay, n)
        # as many arguments as the header declares
        decl = re.search(rf"\b{n}\(([^;]*)\);", txt).group(1)
        want = 0 if decl.strip() == "void" else decl.count(",") + 1
        assert len(LL.SIGNATURES[n][1]) == want, n


def test_header_compiles_as_c_and_constants_match(tmp_path):
    src = tmp_path / "c.c"
    src.write_text('#include <stdio.h>\n#include "muon_layers.h"\nint main(void){printf("%d %d %d %d %d %d",'
                   "MUON_ACT_NONE, MUON_ACT_RELU, MUON_ACT_GELU, MUON_ACT_GELU_TANH, MUON_ACT_SILU,"
                   "MUON_GROUPED_MAX_EXPERTS);return 0;}")
    exe = tmp_path / "c"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    a = LL.ACTIVATIONS
    assert got == [a["none"], a["relu"], a["gelu"], a["gelu_tanh"], a["silu"], LL.MUON_GROUPED_MAX_EXPERTS]


X, Y = 0x1000, 0x2000   # addresses that are checked, never read


def _fwd(lay, **kw):
    a = dict(x=X, ldx=8, w=X, ldw=6, t=0, bias=None, res=None, ldr=6, y=Y, ldy=6, z=None, ldz=6, rows=4, inner=8,
             outer=6, dtype=L.MUON_F32, act=0, ws=None, wsb=0)
    a.update(kw)
    return lay.muon_linear_forward(*a.values(), None)


@pytest.mark.parametrize("kw,word", [
    (dict(x=None), "x is NULL"), (dict(w=None), "w is NULL"), (dict(y=None), "y is NULL"), (dict(rows=-1), "rows"),
    (dict(inner=0), "inner"), (dict(outer=0), "outer"), (dict(outer=1 << 31, ldw=1 << 31), "outer"),
    (dict(ldx=7), "x has leading"), (dict(ldw=5), "w has leading"), (dict(t=1), "w has leading"),
    (dict(ldy=5), "y has leading"), (dict(res=X, ldr=5), "residual"), (dict(z=X, ldz=5), "preact"),
    (dict(x=X + 2), "aligned"), (dict(bias=X + 1), "bias"), (dict(act=5), "activation"), (dict(act=-1), "activation"),
    (dict(ldx=1 << 41), "leading")])
def test_linear_forward_refuses(lay, kw, word):
    assert _fwd(lay, **kw) == L.MUON_ERR_INVALID_ARG
    assert word in lay.muon_layers_last_error().decode()


def test_dtypes_and_small_workspaces_are_refused(lay):
    assert _fwd(lay, dtype=2) == L.MUON_ERR_UNSUPPORTED
    n = ctypes.c_size_t()
    assert lay.muon_linear_workspace_bytes(100, 64, 48, L.MUON_BF16, 2, 1, ctypes.byref(n)) == L.MUON_OK
    assert n.value >= 100 * 48 * 2
    args = [X, 48, X, 64, X, 48, 0, X, 48, Y, 64, Y, 48, Y, 100, 64, 48, L.MUON_BF16, 2]
    assert lay.muon_linear_backward(*args, None, n.value, None) == L.MUON_ERR_INVALID_ARG
    assert lay.muon_linear_backward(*args, 0x1000, n.value - 1, None) == L.MUON_ERR_WORKSPACE_TOO_SMALL
    assert lay.muon_linear_backward(*args, 0x1010, n.value, None) == L.MUON_ERR_INVALID_ARG
    assert lay.muon_linear_workspace_bytes(1, 1, 1, 0, 0, 0, None) == L.MUON_ERR_INVALID_ARG
    assert lay.muon_layer_norm_workspace_bytes(4, 8, ctypes.byref(n)) == L.MUON_OK and n.value >= 2 * 8 * 4
    assert lay.muon_layer_norm_backward(X, 8, X, 8, None, X, X, Y, 8, Y, None, 4, 8, 0, 0, 0x1000, n.value - 1,
                                        None) == L.MUON_ERR_WORKSPACE_TOO_SMALL


def test_workspace_beyond_the_need_must_be_aligned_too(lay):
    """A forward pass that needs no workspace may still use one, for copies of unaligned operands."""
    n = ctypes.c_size_t()
    for flags, some in ((0, False), (2, True)):
        assert lay.muon_linear_workspace_bytes(100, 63, 65, L.MUON_BF16, 0, flags, ctypes.byref(n)) == L.MUON_OK
        assert (n.value > 100 * 63 * 2) == some
    a = [X, 63, X, 65, 0, None, None, 0, Y, 65, None, 0, 100, 63, 65, L.MUON_BF16, 0]
    assert lay.muon_linear_forward(*a, 0x1010, n.value, None) == L.MUON_ERR_INVALID_ARG
    assert "aligned" in lay.muon_layers_last_error().decode()
    assert lay.muon_linear_workspace_bytes(100, 63, 65, L.MUON_BF16, 0, 4, ctypes.byref(n)) == L.MUON_ERR_INVALID_ARG


def test_grouped_refusals(lay):
    ptrs = (ctypes.c_void_p * 3)(X, X, X)
    hole = (ctypes.c_void_p * 3)(X, None, X)

    def call(w=ptrs, experts=3, off=X, rows=4, ldw=6):
        return lay.muon_grouped_linear_forward(X, 8, w, ldw, 0, off, experts, Y, 6, rows, 8, 6, 0, None, 0, None)

    for kw, word in ((dict(w=None), "w is NULL"), (dict(w=hole), "w[1]"), (dict(experts=0), "experts"),
                     (dict(experts=257), "experts"), (dict(off=None), "offsets"), (dict(off=X + 2), "offsets"),
                     (dict(rows=-1), "rows"), (dict(ldw=5), "w has leading")):
        assert call(**kw) == L.MUON_ERR_INVALID_ARG, kw
        assert word in lay.muon_layers_last_error().decode()


def test_layer_norm_refusals(lay):
    def call(x=X, y=Y, ld=8, cols=8, eps=1e-5, dt=0, wdt=0, w=None):
        return lay.muon_layer_norm_forward(x, ld, w, None, y, ld, None, None, 4, cols, eps, dt, wdt, None)

    assert call(dt=3) == L.MUON_ERR_UNSUPPORTED and call(dt=0, wdt=1) == L.MUON_ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(y=None), dict(ld=7), dict(cols=0), dict(eps=float("inf")), dict(eps=-1.0),
               dict(w=X + 1)):
        assert call(**kw) == L.MUON_ERR_INVALID_ARG, kw
    assert lay.muon_layer_norm_backward(X, 8, X, 8, None, None, X, Y, 8, None, None, 4, 8, 0, 0, None, 0,
                                        None) == L.MUON_ERR_INVALID_ARG


def test_last_error_clears_on_success(lay):
    assert _fwd(lay, x=None) != L.MUON_OK and lay.muon_layers_last_error() != b""
    assert _fwd(lay, rows=0, x=None, y=None, w=None) == L.MUON_OK
    assert lay.muon_layers_last_error() == b""


def test_no_layer_kernel_spills(tmp_path):
    lib = open(LL.LIB_PATH, "rb").read()
    seen, bad = 0, {}
    for at in (m.start() for m in re.finditer(b"\x7fELF", lib)):
        if int.from_bytes(lib[at + 18:at + 20], "little") != 224:   # AMDGPU
            continue
        path = tmp_path / f"{at}.co"
        path.write_bytes(lib[at:])
        notes = subprocess.run([READELF, "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        for part in notes.split(".agpr_count:")[1:]:
            name = re.search(r"\.name: +(\S+)", part.split(".private_segment_fixed_size:")[0].split(".max_flat")[-1])
            val = {k: int(re.search(rf"\.{k}: +(\d+)", part).group(1))
                   for k in ("private_segment_fixed_size", "vgpr_spill_count")}
            seen += 1
            if any(val.values()):
                bad[name.group(1)] = val
    assert seen > 10 and not bad, bad
