"""Refusals of the context-free operators that need no device, beyond tests/test_operators_cpu.py."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

import paper_2403_09054_b200 as kf
from tests.test_operators_cpu import FAR, _beam, _norm, _step

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("value", [-1, 2])
def test_packed_step_self_test_argument(value):
    a = _step(debug_fail_first_wait=value)
    assert kf.LIB.kf_packed_scratch_bytes(C.byref(a)) == 0
    assert kf.LIB.kf_decode_step_packed(C.byref(a), *FAR[:8], None, None, None, FAR[11], 1 << 30, None) == kf.KF_EINVAL


def _overlaps(call, sizes, written, base=FAR[1:]):
    """For every pair of which one is written: the second placed on the first's last byte's 256 bytes, or over its start, is refused."""
    for i, a in enumerate(sizes):
        for j, b in enumerate(sizes):
            if i == j or not (i in written or j in written):
                continue
            for at in (base[i] + max(0, a - 1) // 256 * 256, base[i] - max(0, b - 1) // 256 * 256):      # the last 256 bytes of a, or the last of b on a
                p = list(base[:len(sizes)])
                p[j] = at
                assert call(p) == kf.KF_EINVAL, (i, j, hex(at))


def test_packed_step_refuses_what_it_would_write_into_another_tensor():
    slopes = FAR[13]
    a = _step(batch=2, n_heads=8, n_kv_heads=4, head_dim=64, budget_k=32, bias_mode=1, d_alibi_slopes=slopes)
    need = kf.LIB.kf_packed_scratch_bytes(C.byref(a))
    U, d, k = 8, 64, 32
    sizes = [U * k * 80, U * k * 4, U * k * 4, U * 4, 2 * U * d * 2, U * d * 2, U * d * 2, 2 * U * d * 2, U * (k + 1) * 4, U * 4, U * 2 * d * 2, need]
    written = {0, 1, 2, 3, 7, 8, 9, 10, 11}
    _overlaps(lambda p: kf.LIB.kf_decode_step_packed(C.byref(a), *p, need, None), sizes, written)
    for i in written:                                    # the slopes under an output
        p = FAR[:12]
        p[i] = slopes
        assert kf.LIB.kf_decode_step_packed(C.byref(a), *p, need, None) == kf.KF_EINVAL


def test_norm_rotate_refuses_outputs_over_its_inputs():
    a = _norm()                                          # 2 x 3 tokens, 4 + 2 heads of 64
    sizes = [2 * 3 * 512 * 2, 128, 128, 24, 6 * 4 * 64 * 2, 6 * 2 * 64 * 2, 6 * 2 * 64 * 2]
    _overlaps(lambda p: kf.LIB.kf_qk_norm_rotate(C.byref(a), *p, None), sizes, {4, 5, 6})


def test_beam_select_refuses_outputs_over_its_inputs():
    a = _beam(batch=40, beams=3, vocab=1000, row_stride=1000, take=6)
    need = kf.LIB.kf_beam_scratch_bytes(C.byref(a))
    _overlaps(lambda p: kf.LIB.kf_beam_select(C.byref(a), *p, need, None), [120 * 2000, 480, 120, 960, 960, 960, need], {3, 4, 5, 6})
    # between rows that lie apart there is room: only what touches a row is refused
    a = _beam(batch=40, beams=3, vocab=1000, row_stride=4000, take=6)
    need = kf.LIB.kf_beam_scratch_bytes(C.byref(a))
    for off in (0, 1996, 7044, 119 * 8000 + 1996):       # a row's first and last words, the next row's first, the last row's last
        p = FAR[:7]
        p[3] = FAR[0] + off
        assert kf.LIB.kf_beam_select(C.byref(a), *p, need, None) == kf.KF_EINVAL, off


def test_row_conversions_refuse_a_count_that_they_would_overwrite():
    K, V, cache, length = FAR[:4]
    for at in (cache, cache + 2 * 4 * 80 - 4):
        assert kf.LIB.kf_pack_cache(2, 3, 4, 64, K, V, at, cache, None) == kf.KF_EINVAL
    for at in (K, K + 2 * 3 * 128 - 4, V):
        assert kf.LIB.kf_unpack_cache(2, 3, 4, 64, cache, at, K, V, None) == kf.KF_EINVAL


def _python(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)


def test_the_extension_is_loaded_by_the_first_operator_call_only():
    """Importing the package and the context's calls need neither the extension nor a compiler for it; an operator call without it fails loudly."""
    r = _python("""
import sys, os
import paper_2403_09054_b200 as kf
from paper_2403_09054_b200 import binding
assert "_kf_torch" not in sys.modules and type(binding._kf_torch) is binding._TorchSide
cfg, keep = kf.make_config(n_layers=1, batch=1, n_heads=1, head_dim=64, budget_k=4, recent_w=1, max_prompt_len=8, gen_len_T=1)
assert kf.kf_workspace_bytes(cfg) > 0 and kf.kf_packed_slot_bytes(64) == 80
os.environ["CXX"] = "false"
here = binding._build.torch_lib
binding._build.torch_lib = lambda: here() + ".none"
try:
    kf.kf_pack_cache(K=None, V=None, cache=None)
except Exception as e:
    print(type(e).__name__)
binding._build.torch_lib = here
try:
    kf.kf_pack_cache(K=None, V=None, cache=None)
except ValueError:
    print("refused by", type(binding._kf_torch).__name__)
""")
    assert r.returncode == 0, r.stderr
    assert r.stdout.split("\n")[:2] == ["CalledProcessError", "refused by module"], r.stdout


def test_the_extension_is_one_of_the_installed_torch():
    assert f"torch-{torch.__version__}." in kf.binding._build.torch_lib()
