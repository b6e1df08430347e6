"""The AdamW library's C ABI and its Python entry points without a GPU: exports,
bindings, and argument checks, which come before any device call."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2606_27153_amd import AdamW, adamw
from paper_2606_27153_amd import _adamw_lib as AL
from paper_2606_27153_amd import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "muon_adamw.h")
X = 0x1000   # an address that is checked, never read


@pytest.fixture(scope="module")
def lib():
    return AL.load()


def test_every_declared_function_is_exported_and_bound(lib):
    txt = open(HEADER).read()
    names = sorted(set(re.findall(r"^MUON_API\s+[\w\s\*]+?\b(muon_\w+)\(", txt, flags=re.M)))
    assert names == sorted(AL.SIGNATURES)
    for n in names:
        assert hasattr(lib, n)
        decl = re.search(rf"\b{n}\(([^;]*)\);", txt).group(1)
        assert len(AL.SIGNATURES[n][1]) == (0 if decl.strip() == "void" else decl.count(",") + 1), n


def test_header_compiles_as_c_and_structures_match(tmp_path):
    src = tmp_path / "c.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "muon_adamw.h"\nint main(void){'
                   'printf("%zu %zu %zu %zu %d", sizeof(muon_adamw_tensor), offsetof(muon_adamw_tensor, step),'
                   "offsetof(muon_adamw_tensor, grad_dtype), sizeof(muon_adamw_opts), MUON_ADAMW_BLOCK);return 0;}")
    exe = tmp_path / "c"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    t = AL.muon_adamw_tensor
    assert got == [ctypes.sizeof(t), t.step.offset, t.grad_dtype.offset, ctypes.sizeof(AL.muon_adamw_opts),
                   AL.MUON_ADAMW_BLOCK]
    assert ctypes.sizeof(t) == 8 * 8    # the words that adamw_step fills


def _step(lib, tensor=None, opts=None, count=1):
    t = dict(param=X, grad=X, exp_avg=X, exp_avg_sq=X, bases=X, n=4, step=1, param_dtype=0, grad_dtype=0)
    t.update(tensor or {})
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, state_bits=32, seed=0)
    o.update(opts or {})
    return lib.muon_adamw_step(ctypes.byref(AL.muon_adamw_tensor(**t)), count,
                               ctypes.byref(AL.muon_adamw_opts(**o)), None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("tensor,opts,word", [
    (dict(param=None), {}, "param"), (dict(exp_avg=None), {}, "exp_avg"), (dict(exp_avg_sq=None), {}, "exp_avg_sq"),
    (dict(param=X + 2), {}, "aligned"), (dict(grad=X + 1), {}, "aligned"), (dict(exp_avg=X + 2), {}, "aligned"),
    (dict(bases=None), dict(state_bits=8), "bases"), (dict(bases=X + 1), dict(state_bits=8), "aligned"),
    (dict(n=-1), {}, "n -1"), (dict(n=1 << 41), {}, "n "), (dict(step=0), {}, "step"), (dict(step=-5), {}, "step"),
    ({}, dict(lr=-1.0), "lr"), ({}, dict(lr=NAN), "lr"), ({}, dict(lr=INF), "lr"), ({}, dict(beta1=1.0), "beta1"),
    ({}, dict(beta1=-0.1), "beta1"), ({}, dict(beta2=1.0), "beta2"), ({}, dict(beta2=NAN), "beta2"),
    ({}, dict(eps=-1.0), "eps"), ({}, dict(eps=INF), "eps"), ({}, dict(weight_decay=-1.0), "weight_decay"),
    ({}, dict(weight_decay=INF), "weight_decay")])
def test_step_refuses(lib, tensor, opts, word):
    assert _step(lib, tensor, opts) == L.MUON_ERR_INVALID_ARG
    assert word in lib.muon_adamw_last_error().decode()


def test_types_are_refused_and_nothing_is_fine(lib):
    assert _step(lib, dict(param_dtype=2)) == L.MUON_ERR_UNSUPPORTED
    assert _step(lib, dict(grad_dtype=-1)) == L.MUON_ERR_UNSUPPORTED
    assert _step(lib, None, dict(state_bits=16)) == L.MUON_ERR_UNSUPPORTED
    assert lib.muon_adamw_step(None, 1, ctypes.byref(AL.muon_adamw_opts(1e-3, 0.9, 0.99, 0, 0, 32, 0)), None) == \
        L.MUON_ERR_INVALID_ARG
    assert lib.muon_adamw_step(None, 0, None, None) == L.MUON_ERR_INVALID_ARG
    # no tensors, no elements, no gradient: nothing to do, nothing is launched
    assert _step(lib, count=0) == L.MUON_OK and lib.muon_adamw_last_error() == b""
    assert _step(lib, dict(n=0, param=None)) == L.MUON_OK
    assert _step(lib, dict(grad=None, param=None)) == L.MUON_OK
    assert _step(lib, count=-1) == L.MUON_ERR_INVALID_ARG
    assert lib.muon_adamw_state_values(X, X, X, -1, X, X, None) == L.MUON_ERR_INVALID_ARG
    assert lib.muon_adamw_state_values(X, X, None, 4, X, X, None) == L.MUON_ERR_INVALID_ARG
    assert lib.muon_adamw_state_values(X, X, X, 4, X + 1, X, None) == L.MUON_ERR_INVALID_ARG
    assert lib.muon_adamw_state_values(X, X, X, 4, None, None, None) == L.MUON_OK


def test_python_refusals():
    p = torch.zeros(8)
    with pytest.raises(ValueError, match="GPU"):
        adamw.adamw_step([p], [p], [adamw.new_state(p)], step=1, lr=1e-3)
    with pytest.raises(ValueError, match="1 params"):
        adamw.adamw_step([p], [], [adamw.new_state(p)], step=1, lr=1e-3)
    with pytest.raises(TypeError, match="param 0"):
        adamw.adamw_step([3], [p], [adamw.new_state(p)], step=1, lr=1e-3)
    with pytest.raises(ValueError, match="bits"):
        adamw.new_state(p, 16)
    with pytest.raises(ValueError, match="GPU"):
        adamw.state_values(adamw.new_state(p, 8))
    with pytest.raises(TypeError):
        adamw.state_values(3)
    assert adamw.adamw_step([], [], [], step=1, lr=1e-3) is None
    for kw in (dict(lr=-1.0), dict(betas=(0.9, 1.0)), dict(betas=(0.9,)), dict(eps=-1), dict(weight_decay=-1),
               dict(state_bits=4), dict(lr=NAN)):
        with pytest.raises(ValueError):
            AdamW([torch.nn.Parameter(torch.zeros(2))], **kw)


def test_binding_gives_nothing_for_tensors_that_do_not_fit():
    """What it answers with None is then named by the checks one by one."""
    f, p = AL.tensors(), torch.zeros(3)
    for args in (([p], [p], [(p, p)], [1]), (1, 2, 3, 4), ([None], [None], [None], [1]), ([p], [], [(p, p)], [1]),
                 ([p], [p], [p], [1]), ([p.to_sparse()], [p], [(p, p)], [1])):
        assert f(*args) is None
    with pytest.raises(TypeError):
        f([p])


def test_states_keep_their_types_through_a_state_dict():
    p, q = torch.nn.Parameter(torch.zeros(300, dtype=torch.bfloat16)), torch.nn.Parameter(torch.zeros(5))
    for bits in (32, 8):
        opt = AdamW([p, q], state_bits=bits)
        for t in (p, q):
            opt.state[t] = dict(zip(("step", "exp_avg", "exp_avg_sq", "bases"), (3, *adamw.new_state(t, bits))))
        opt.state[p]["exp_avg"][7] = 200 if bits == 8 else 1 + 2.0 ** -20
        if bits == 8:
            opt.state[p]["bases"][1, 0] = 1901
        fresh = AdamW([p, q], state_bits=bits)
        fresh.load_state_dict(opt.state_dict())
        for t in (p, q):
            for k, v in opt.state[t].items():
                got = fresh.state[t][k]
                assert got == v if k == "step" else got.dtype == v.dtype and torch.equal(got, v), k
                assert k == "step" or got.data_ptr() != v.data_ptr()


def test_a_refused_step_does_not_count():
    p = torch.nn.Parameter(torch.zeros(8))
    p.grad = torch.zeros(8)
    opt = AdamW([p])
    for _ in range(2):
        with pytest.raises(ValueError, match="GPU"):
            opt.step()
    assert opt.state[p]["step"] == 0


def test_written_tensors_get_another_version():
    p, q, m, v = (torch.zeros(3) for _ in range(4))
    with torch.inference_mode():
        inside = torch.zeros(3)     # (without a version)
    AL.written([p, q, inside], (p, None, p), [(m, v), [q, q], [inside, inside]])
    assert p._version > 0 and m._version > 0 and v._version > 0 and q._version == 0
    AL.written([], [], [])
    with pytest.raises(TypeError):
        AL.written(1, 2, 3)
    with pytest.raises(TypeError):
        AL.written([p], [p], [4])


def test_a_state_that_cannot_be_made_leaves_none():
    """A group's own options are read at the step: what is wrong with them is said every time."""
    p = torch.nn.Parameter(torch.zeros(8))
    p.grad = torch.zeros(8)
    opt = AdamW([dict(params=[p], state_bits=4)])
    for _ in range(2):
        with pytest.raises(ValueError, match="4 bits"):
            opt.step()
        assert not opt.state[p]
