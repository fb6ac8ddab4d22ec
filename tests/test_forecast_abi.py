"""Host-side checks of the forecasting operators' C ABI that need no GPU: exports, layouts, workspace
sizes and refusals (everything is validated before anything is launched)."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def F():
    from paper_2407_14843_b200 import build
    build.build_library()
    from paper_2407_14843_b200 import forecast
    return forecast


def test_every_declared_function_is_exported(F):
    header = open(os.path.join(ROOT, "include", "themis_forecast.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    assert set(re.findall(r"\b(themis_[a-z0-9_]+)\s*\(", header)) == set(F.EXPORTS)
    lib = ctypes.CDLL(F.solver.LIB_PATH)
    for name in F.EXPORTS:
        assert hasattr(lib, name), name


def test_header_is_plain_c_and_layouts_match(F, tmp_path):
    src = tmp_path / "use_forecast.c"
    src.write_text(r'''
#include <stdio.h>
#include <string.h>
#include "themis_forecast.h"
int main(void) {
    themis_ssm_problem_t p;
    themis_linear_problem_t l;
    size_t bytes = 1;
    int32_t count = 0;
    memset(&p, 0, sizeof p);
    p.batch = 2; p.length = 100; p.channels = 64; p.state = 16; p.groups = 1; p.conv_width = 4; p.dtype = THEMIS_DTYPE_BF16;
    if (themis_ssm_workspace_bytes(&p, 1, &bytes) != THEMIS_OK || bytes == 0) return 1;
    if (themis_ssm_checkpoints(&p, &count) != THEMIS_OK || count != (100 + THEMIS_SSM_CHUNK - 1) / THEMIS_SSM_CHUNK) return 2;
    memset(&l, 0, sizeof l);
    l.rows = 100; l.out_features = 64; l.in_features = 64; l.dtype = THEMIS_DTYPE_F16;
    l.x_row = l.weight_row = l.residual_row = l.dy_row = 64;
    if (themis_linear_workspace_bytes(&l, 0, 0, &bytes) != THEMIS_OK || bytes != 0) return 3;
    printf("%zu %zu %zu %zu %zu %d\n", sizeof(themis_ssm_problem_t), sizeof(themis_ssm_inputs_t), sizeof(themis_ssm_outputs_t),
           sizeof(themis_ssm_grads_t), sizeof(themis_linear_problem_t), THEMIS_SSM_CHUNK);
    return 0;
}
''')
    exe = tmp_path / "use_forecast"
    lib_dir = os.path.dirname(F.solver.LIB_PATH)
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                           "-o", str(exe), "-L", lib_dir, "-l:libthemis.so", f"-Wl,-rpath,{lib_dir}"])
    sizes = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    classes = (F.SsmProblem, F.SsmInputs, F.SsmOutputs, F.SsmGrads, F.LinearProblem)
    assert sizes == [ctypes.sizeof(c) for c in classes] + [F.SSM_CHUNK]
    assert [s.size for s in (F._PROBLEM, F._INPUTS, F._OUTPUTS, F._GRADS, F._LINEAR)] == sizes[:5]


def ssm(F, **kw):
    p = F.SsmProblem(2, 100, 64, 16, 1, 4, 1, 0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), -1), (dict(length=-1), -1), (dict(channels=0), -1), (dict(state=0), -1), (dict(groups=0), -1),
    (dict(groups=3), -1), (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(flags=1), -1), (dict(x_row=-1), -1), (dict(c_group=-8), -1),
    (dict(state=65), -2), (dict(conv_width=1), -2), (dict(conv_width=5), -2), (dict(channels=65536), -2),
])
def test_invalid_scans_are_refused(F, kw, code):
    p = ssm(F, **kw)
    n = ctypes.c_size_t()
    assert F._lib.themis_ssm_workspace_bytes(bytes(p), 0, ctypes.byref(n)) == code
    for call in (lambda: F._lib.themis_ssm_forward(bytes(p), None, None, None, 0, None), lambda: F._lib.themis_ssm_step(bytes(p), None, None, None),
                 lambda: F._lib.themis_ssm_backward(bytes(p), None, None, None, None, None, 0, None)):
        assert call() == code


def test_scan_pointers_and_workspaces_are_checked(F):
    one = 256
    full = [one] * 13
    def inputs(**kw):
        v = dict(zip((f[0] for f in F.SsmInputs._fields_), full))
        v.update(kw)
        return F._INPUTS.pack(*v.values())
    p = bytes(ssm(F, length=4096))
    out = F._OUTPUTS.pack(one, 512, 512, 512)
    need = F.themis_ssm_workspace_bytes(p, False)
    assert need > 0 and F.themis_ssm_workspace_bytes(bytes(ssm(F, length=0)), True) == 0
    fwd = F._lib.themis_ssm_forward
    assert fwd(p, None, out, one, need, None) == F.E_INVALID_ARG
    for name in ("x", "dt", "b", "c", "a", "conv_weight"):
        assert fwd(p, inputs(**{name: 0}), out, one, need, None) == F.E_INVALID_ARG, name
    assert fwd(p, inputs(), F._OUTPUTS.pack(0, 512, 512, 512), one, need, None) == F.E_INVALID_ARG
    assert fwd(p, inputs(), F._OUTPUTS.pack(one, one, 512, 512), one, need, None) == F.E_INVALID_ARG      # states in place
    assert fwd(p, inputs(), F._OUTPUTS.pack(one, 512, one, 512), one, need, None) == F.E_INVALID_ARG
    assert fwd(p, inputs(), out, None, need, None) == F.E_INVALID_ARG
    assert fwd(p, inputs(), out, one + 8, need, None) == F.E_INVALID_ARG
    assert fwd(p, inputs(), out, one, need - 1, None) == F.E_WORKSPACE_TOO_SMALL
    bwd, grads, back = F._lib.themis_ssm_backward, F._GRADS.pack(*[one] * 10), F.themis_ssm_workspace_bytes(p, True)
    assert bwd(p, inputs(), None, one, grads, one, back, None) == F.E_INVALID_ARG
    assert bwd(p, inputs(), one, None, grads, one, back, None) == F.E_INVALID_ARG
    assert bwd(p, inputs(z=0), one, one, grads, one, back, None) == F.E_INVALID_ARG                       # dz without z
    assert bwd(p, inputs(), one, one, grads, one, back - 1, None) == F.E_WORKSPACE_TOO_SMALL
    step = F._lib.themis_ssm_step
    assert step(p, inputs(conv_state=0), out, None) == F.E_INVALID_ARG
    assert step(p, inputs(ssm_state=0), out, None) == F.E_INVALID_ARG
    assert step(p, inputs(), F._OUTPUTS.pack(one, 0, one, 0), None) == F.E_INVALID_ARG
    assert step(bytes(ssm(F, batch=2 ** 31 - 1, channels=65535)), inputs(), out, None) == F.E_UNSUPPORTED_SIZE


def linear(F, **kw):
    p = F.LinearProblem(100, 64, 48, 1, 0, 0, 48, 48, 64, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), -1), (dict(out_features=0), -1), (dict(in_features=0), -1), (dict(dtype=0), -1), (dict(dtype=3), -1),
    (dict(activation=4), -1), (dict(activation=-1), -1), (dict(flags=2), -1), (dict(x_row=47), -1), (dict(weight_row=47), -1),
    (dict(residual_row=63), -1), (dict(dy_row=63), -1), (dict(rows=2 ** 30 + 1), -2),
    (dict(out_features=2 ** 24 + 1, residual_row=2 ** 25, dy_row=2 ** 25), -2), (dict(in_features=2 ** 24 + 1, x_row=2 ** 25, weight_row=2 ** 25), -2),
])
def test_invalid_products_are_refused(F, kw, code):
    p = linear(F, **kw)
    n = ctypes.c_size_t()
    assert F._lib.themis_linear_workspace_bytes(bytes(p), 0, 0, ctypes.byref(n)) == code
    assert F._lib.themis_linear_forward(bytes(p), *[None] * 8, 0, None) == code
    assert F._lib.themis_linear_backward(bytes(p), *[None] * 9, 0, None) == code


def test_product_pointers_and_workspaces_are_checked(F):
    p = bytes(linear(F, activation=2))
    fwd, bwd = F._lib.themis_linear_forward, F._lib.themis_linear_backward
    assert F.themis_linear_workspace_bytes(p, False) == 0                    # aligned operands are read where they are
    assert F.themis_linear_workspace_bytes(p, False, True) > 0
    assert F.themis_linear_workspace_bytes(bytes(linear(F, x_row=49)), False) > 0
    assert F.themis_linear_workspace_bytes(bytes(linear(F, rows=0)), True) == 0
    one = 256
    for missing in (0, 1, 4):                                                # x, weight, y
        args = [one] * 6
        args[missing] = None
        assert fwd(p, *args, None, None, 0, None) == F.E_INVALID_ARG
    assert fwd(p, one + 2, one, None, None, one, None, None, None, 0, None) == F.E_INVALID_ARG          # unaligned, no workspace
    need = F.themis_linear_workspace_bytes(p, True)
    assert bwd(p, one, one, one, None, one, one, one, None, one, need, None) == F.E_INVALID_ARG         # no pre
    assert bwd(p, None, one, one, one, one, one, one, None, one, need, None) == F.E_INVALID_ARG
    assert bwd(p, one, None, one, one, None, one, None, None, one, need, None) == F.E_INVALID_ARG       # dweight without x
    assert bwd(p, one, one, one, one, one, one, one, None, one, need - 1, None) == F.E_WORKSPACE_TOO_SMALL
    assert bwd(p, one, one, one, one, one, one, one, None, one + 8, need, None) == F.E_INVALID_ARG


def test_calls_on_cpu_tensors_are_refused(F):
    import torch
    x, w = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(8, 16, dtype=torch.bfloat16)
    with pytest.raises((TypeError, ValueError)):
        F.linear(x, w)
    d = torch.zeros(2, 3, 8)
    with pytest.raises((TypeError, ValueError)):
        F.ssm_scan(d, d, torch.zeros(8, 4), torch.zeros(2, 3, 4), torch.zeros(2, 3, 4), torch.zeros(8, 4))


def test_an_expired_wait_is_raised_by_the_next_call(F, monkeypatch):
    """The host's side, with the device's write made by the test."""
    import torch
    F.check_status()
    monkeypatch.setattr(F, "_status_word", ctypes.c_int32(F.STATUS_TIMEOUT))
    with pytest.raises(F.WaitExpired):
        F.check_status()
    F.check_status()                                                         # raised once
    word = torch.zeros(1, dtype=torch.int32)
    monkeypatch.setattr(F, "_status_memory", word)
    monkeypatch.setattr(F, "_status_word", ctypes.c_int32.from_address(word.data_ptr()))
    assert F._status(None, 0) == word.data_ptr()
    word[0] = F.STATUS_TIMEOUT
    with pytest.raises(F.WaitExpired):
        F._status(None, 0)
    assert word.item() == 0


def test_lengths_that_leave_no_room_to_round_up_are_refused(F):
    """Times are counted in 32 bits, up to the next multiple of a part."""
    n, count = ctypes.c_size_t(), ctypes.c_int32()
    for length, code in ((2 ** 30, F.OK), (2 ** 30 + 1, F.E_UNSUPPORTED_SIZE), (2 ** 31 - 1, F.E_UNSUPPORTED_SIZE)):
        p = bytes(ssm(F, batch=1, length=length, channels=1, state=1))
        assert F._lib.themis_ssm_checkpoints(p, ctypes.byref(count)) == code
        assert F._lib.themis_ssm_workspace_bytes(p, 0, ctypes.byref(n)) == code
        assert F._lib.themis_ssm_workspace_bytes(p, 1, ctypes.byref(n)) == code
        if code == F.OK:
            assert count.value == length // F.SSM_CHUNK
    # a step has no use for it
    assert F._lib.themis_ssm_step(bytes(ssm(F, batch=0, length=2 ** 31 - 1)), F._INPUTS.pack(*[0] * 13), F._OUTPUTS.pack(*[0] * 4), None) == F.OK
