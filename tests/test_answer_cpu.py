"""Refusals of the answer operators (8-bit products, token probabilities, draft
verification), on the host: every call below is refused before it would touch a
device, with the documented code and a message. Pointers are never read."""

from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2606_18600_amd import build, int8, speculate
from paper_2606_18600_amd import stage as S
from tests.test_abi_cpu import ROOT, _lib

A, B, C, D = 0x10000, 0x20000, 0x30000, 0x40000   # 16-byte aligned, never dereferenced
INV, UNS, CAP = S.STAGE_ERR_INVALID_ARG, S.STAGE_ERR_UNSUPPORTED, S.STAGE_ERR_CAPACITY
F32, BF16 = S.STAGE_F32, S.STAGE_BF16


def _refused(code, want):
    assert code == want, (code, S.stage_last_error())
    assert S.stage_last_error()


def test_quant_bytes():
    _lib()
    # values in strips of 16 rows, k padded to 128, a scale per padded row
    assert S.stage_quant_bytes(1, 1) == 16 * 128 + 16 * 4
    assert S.stage_quant_bytes(17, 129) == 32 * 256 + 32 * 4
    assert S.stage_quant_bytes(128256, 8192) == 128256 * 8192 + 128256 * 4
    assert S.stage_quant_bytes(0, 64) == 0
    for rows, k in ((-1, 64), (4, 0), (4, 131073), ((1 << 21) + 1, 64)):
        assert S.stage_quant_bytes(rows, k) == 0


@pytest.mark.parametrize("args,code", [
    ((2, A, 64, 4, 64, B), UNS),            # no such type
    ((F32, A, 64, -1, 64, B), INV),
    ((F32, A, 64, 4, 0, B), INV),
    ((F32, A, 1 << 18, 4, 131073, B), UNS),  # int32 sums could overflow
    ((F32, A, 63, 4, 64, B), INV),          # row stride below the row's length
    ((F32, A, -64, 4, 64, B), INV),
    ((F32, A, 1 << 50, 4, 64, B), INV),
    ((F32, 0, 64, 4, 64, B), INV),
    ((F32, A, 64, 4, 64, 0), INV),
    ((F32, A + 2, 64, 4, 64, B), INV),      # fp32 at an odd address
    ((BF16, A + 1, 64, 4, 64, B), INV),
    ((BF16, A, 64, 4, 64, B + 8), INV),
])
def test_quant_rows_refuses(args, code):
    _refused(_lib().stage_quant_rows(*args, None), code)


@pytest.mark.parametrize("args,code", [
    ((A, 64, B, -1, 64, C), INV), ((0, 64, B, 4, 64, C), INV), ((A, 64, 0, 4, 64, C), INV),
    ((A, 64, B + 2, 4, 64, C), INV), ((A, 63, B, 4, 64, C), INV), ((A, 64, B, 4, 64, C + 4), INV),
    ((A, 64, B, 4, 1 << 20, C), UNS),
])
def test_quant_pack_refuses(args, code):
    _refused(_lib().stage_quant_pack(*args, None), code)


@pytest.mark.parametrize("args,code", [
    ((A, 4, B, 8, 64, 5, C, 8), UNS), ((A, -4, B, 8, 64, F32, C, 8), INV),
    ((A, 4, B, -8, 64, F32, C, 8), INV), ((A, 4, B, 8, 0, F32, C, 8), INV),
    ((A, 4, B, 8, 64, F32, C, 7), INV), ((0, 4, B, 8, 64, F32, C, 8), INV),
    ((A, 4, 0, 8, 64, F32, C, 8), INV), ((A, 4, B, 8, 64, F32, 0, 8), INV),
    ((A + 4, 4, B, 8, 64, F32, C, 8), INV), ((A, 4, B, 8, 64, F32, C + 2, 8), INV),
    ((A, 4, B, 8, 200000, F32, C, 8), UNS),
])
def test_quant_product_refuses(args, code):
    _refused(_lib().stage_quant_product(*args, None, 0, None), code)


@pytest.mark.parametrize("args,code", [
    ((7, A, 64, 4, 64, B, 8, F32, C, 8), UNS), ((F32, A, 64, 4, 64, B, 8, 7, C, 8), UNS),
    ((F32, A, 64, -4, 64, B, 8, F32, C, 8), INV), ((F32, A, 64, 4, 64, B, -8, F32, C, 8), INV),
    ((F32, A, 64, 4, 0, B, 8, F32, C, 8), INV), ((F32, A, 63, 4, 64, B, 8, F32, C, 8), INV),
    ((F32, 0, 64, 4, 64, B, 8, F32, C, 8), INV), ((F32, A + 2, 64, 4, 64, B, 8, F32, C, 8), INV),
    ((F32, A, 64, 4, 64, 0, 8, F32, C, 8), INV), ((F32, A, 64, 4, 64, B + 8, 8, F32, C, 8), INV),
    ((F32, A, 64, 4, 64, B, 8, F32, 0, 8), INV), ((F32, A, 64, 4, 64, B, 8, F32, C, 7), INV),
    ((F32, A, 1 << 18, 4, 131073, B, 8, F32, C, 8), UNS),
])
def test_quant_linear_refuses(args, code):
    _refused(_lib().stage_quant_linear(*args, D, 1 << 20, None), code)


def test_quant_linear_checks_its_workspace():
    lib = _lib()
    need = S.stage_quant_linear_bytes(128, 1280, 8192)
    assert need >= S.stage_quant_bytes(128, 8192) + S.stage_quant_product_bytes(128, 1280, 8192)
    assert S.stage_quant_linear_bytes(4, 0, 64) == 0 == S.stage_quant_linear_bytes(4, 8, -1)
    for ws, size, code in ((0, need, INV), (D, need - 1, CAP), (D + 8, need, INV)):
        _refused(lib.stage_quant_linear(F32, A, 8192, 128, 8192, B, 1280, F32, C, 1280, ws, size,
                                        None), code)


def test_empty_calls_do_nothing():
    lib = _lib()
    assert lib.stage_quant_rows(F32, None, 0, 0, 64, None, None) == S.STAGE_OK
    assert lib.stage_quant_pack(None, 0, None, 0, 64, None, None) == S.STAGE_OK
    assert lib.stage_quant_product(None, 0, None, 8, 64, F32, None, 8, None, 0,
                                   None) == S.STAGE_OK
    assert lib.stage_quant_product(None, 8, None, 0, 64, F32, None, 0, None, 0,
                                   None) == S.STAGE_OK
    assert lib.stage_quant_linear(F32, None, 64, 0, 64, None, 8, F32, None, 8, None, 0,
                                  None) == S.STAGE_OK
    assert lib.stage_token_probs(F32, None, 0, 0, 64, None, F32, None, 0, None, 0,
                                 None) == S.STAGE_OK
    empty = S.stage_drafts(F32, 64, 0, 0, 4)
    assert lib.stage_verify_drafts(ctypes.byref(empty), None, None, None, 0, None) == S.STAGE_OK


def test_lm_head_quant_refuses():
    lib = _lib()
    _refused(lib.stage_lm_head_quant(None, A, B, 1000, C, 4, None, 4, D, None), INV)
    _refused(lib.stage_lm_head_quant(None, A, B + 4, 1000, C, 4, None, 4, D, None), INV)
    _refused(lib.stage_lm_head_quant(None, A, B, (1 << 21) + 1, C, 4, None, 4, D, None), UNS)


@pytest.mark.parametrize("args,code", [
    ((3, A, 64, 2, 64, C, F32, B, 64), UNS), ((F32, A, 64, 2, 64, C, 3, B, 64), UNS),
    ((F32, A, 64, -2, 64, C, F32, B, 64), INV), ((F32, A, 64, 2, 0, C, F32, B, 64), INV),
    ((F32, A, 63, 2, 64, C, F32, B, 64), INV), ((F32, A, 64, 2, 64, C, F32, B, 63), INV),
    ((F32, 0, 64, 2, 64, C, F32, B, 64), INV), ((F32, A, 64, 2, 64, C, F32, 0, 64), INV),
    ((F32, A, 64, 2, 64, C + 2, F32, B, 64), INV),
    ((F32, A, 64, 2, 64, C, BF16, A, 64), INV),      # in place at another type
    ((F32, A, 64, 2, 64, C, F32, A, 80), INV),       # ... and at another stride
    ((F32, A, 1 << 31, 2, (1 << 30) + 1, C, F32, B, 1 << 31), UNS),
])
def test_token_probs_refuses(args, code):
    _refused(_lib().stage_token_probs(*args, D, 1 << 20, None), code)


def test_workspaces_are_checked():
    lib = _lib()
    need = S.stage_quant_product_bytes(128, 1280, 8192)   # a product over several k ranges
    assert need > 0 and S.stage_quant_product_bytes(0, 1280, 8192) == 0
    assert S.stage_quant_product_bytes(4, 8, 0) == 0
    for ws, size, code in ((0, need, INV), (D, need - 1, CAP), (D + 8, need, INV)):
        _refused(lib.stage_quant_product(A, 128, B, 1280, 8192, F32, C, 1280, ws, size, None), code)
    need = S.stage_token_probs_bytes(2, 100000)
    assert need > 0 and S.stage_token_probs_bytes(2, 0) == 0
    for ws, size, code in ((0, need, INV), (D, need - 1, CAP), (D + 8, need, INV)):
        _refused(lib.stage_token_probs(F32, A, 100000, 2, 100000, None, F32, B, 100000, ws, size,
                                       None), code)
    d = S.stage_drafts(F32, 100000, 2, 3, 4, A, 100000, B, 100000, C, C, C, C)
    need = S.stage_verify_bytes(2, 100000)
    assert need > 0 and S.stage_verify_bytes(-1, 64) == 0
    for ws, size, code in ((0, need, INV), (D, need - 1, CAP), (D + 8, need, INV)):
        _refused(lib.stage_verify_drafts(ctypes.byref(d), A, B, ws, size, None), code)


@pytest.mark.parametrize("field,value,code", [
    ("dtype", 9, UNS), ("vocab", 0, INV), ("vocab", (1 << 30) + 1, UNS), ("num_seqs", -1, INV),
    ("num_seqs", 65536, CAP), ("num_drafts", -1, INV), ("num_drafts", (1 << 31) - 2, CAP),
    ("max_drafts", -1, INV), ("max_drafts", (1 << 24) + 1, CAP),
    ("max_drafts", (1 << 31) - 1, CAP), ("target_probs", 0, INV), ("target_probs", A + 2, INV),
    ("ld_target", 63, INV), ("ld_draft", 63, INV), ("draft_probs", B + 1, INV), ("drafts", 0, INV),
    ("drafts", C + 2, INV), ("starts", 0, INV), ("accept_u", 0, INV), ("sample_u", 0, INV),
    ("sample_u", C + 1, INV),
])
def test_verify_drafts_refuses(field, value, code):
    d = S.stage_drafts(F32, 64, 2, 3, 4, A, 64, B, 64, C, C, C, C)
    setattr(d, field, value)
    _refused(_lib().stage_verify_drafts(ctypes.byref(d), A, B, D, 1 << 20, None), code)


def test_verify_drafts_refuses_missing_outputs():
    lib = _lib()
    d = S.stage_drafts(F32, 64, 2, 3, 4, A, 64, B, 64, C, C, C, C)
    _refused(lib.stage_verify_drafts(None, A, B, D, 1 << 20, None), INV)
    _refused(lib.stage_verify_drafts(ctypes.byref(d), None, B, D, 1 << 20, None), INV)
    _refused(lib.stage_verify_drafts(ctypes.byref(d), A, None, D, 1 << 20, None), INV)


def _code(f, *args, **kw):
    with pytest.raises(S.StageError) as e:
        f(*args, **kw)
    return e.value.code


def test_tensor_calls_refuse():
    """The torch-side checks: types, shapes, and tensors that are not on a GPU."""
    x, h = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.float16)
    w = int8.Matrix(torch.zeros(S.stage_quant_bytes(8, 64), dtype=torch.uint8), 8, 64)
    odd = int8.Matrix(w.data, 8, 65)
    assert _code(int8.quantize, x) == INV                  # on the CPU
    assert _code(int8.quantize, h) == UNS
    assert _code(int8.linear, x, odd) == INV               # depths differ
    assert _code(int8.linear, torch.zeros(()), w) == INV
    assert _code(int8.product, w, odd) == INV
    assert _code(int8.product, w, w) == INV
    assert _code(int8.pack_weight, x, torch.zeros(4)) == INV
    assert _code(int8.pack_weight, x.to(torch.int8), torch.zeros(5)) == INV
    assert _code(int8.pack_weight, x.to(torch.int8), torch.zeros(4)) == INV
    assert _code(speculate.token_probs, x) == INV
    assert _code(speculate.token_probs, h) == UNS
    assert _code(speculate.token_probs, x, dtype=torch.float16) == UNS
    i, u = torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    args = [torch.zeros(5, 64), torch.zeros(3, 64), i, i, 4, u, u[:2]]
    assert _code(speculate.verify_drafts, *args) == INV    # on the CPU
    assert _code(speculate.verify_drafts, h, *args[1:]) == UNS
    assert _code(speculate.verify_drafts, *args[:2], i.view(3, 1), *args[3:]) == INV


def test_sizes_beyond_32_bits_are_refused():
    """They would be cut to their low bits on the way into the library."""
    long = torch.zeros(1, 1).expand((1 << 32) + 1, 1)
    assert _code(int8.rows_of, long, "x") == UNS
    assert _code(int8.rows_of, long.t(), "x") == UNS
    assert _code(int8.rows_of, torch.zeros(2, 3, 0), "x") == INV


def test_product_plans(tmp_path):
    """The rule that picks a product's kernel, over 20000 sizes (host code, built with
    g++ against a stand-in of the HIP header): ranges cover k exactly and none is
    empty, their lengths fit the kernel, grids and planes stay within their limits."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "quant_plan_check")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "tests", "host", "include"),
                        os.path.join(ROOT, "tests", "host", "quant_plan_check.cpp"),
                        os.path.join(build.SRC, "quant_plan.cpp"), "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "plans passed" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


def test_matrix_instructions_are_not_masked(tmp_path):
    """A matrix instruction ignores the lane mask, so one inside a divergent branch runs
    for the lanes that did not take it, unless the branch is skipped where no lane
    takes it. The conditions around the products of csrc/k_quant.hip are scalar: in
    the built code no instruction follows a mask without such a skip."""
    out = str(tmp_path / "k_quant.s")
    r = subprocess.run([build.hipcc(), *build.HIPCC_FLAGS, "-x", "hip", "--cuda-device-only", "-S",
                        os.path.join(build.SRC, "k_quant.hip"), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    masked, products = False, 0
    for line in open(out):
        if "s_and_saveexec" in line:
            masked = True
        elif "s_cbranch_execz" in line or "s_or_b64 exec" in line or line.startswith(".LBB"):
            masked = False
        elif "v_mfma_i32" in line:
            products += 1
            assert not masked, line
    assert products > 1000
