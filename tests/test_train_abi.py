"""CPU-side checks of the training operators' C ABI: exported symbols, refusals on the host, work lists and buckets.  No GPU work."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2503_05931_amd import binding, training as T
from tests import train_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E, U = binding.AED_EINVAL, binding.AED_EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2503_05931_amd import build
        build.build()
    return T._lib()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "aed_train.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(aed_[a-z_0-9]+)\s*\(", text)))
    assert sorted(T.EXPORTS) == names and len(names) == 11
    for n in names:
        assert hasattr(lib, n), n


def config(**over):
    c = T.AedAttnConfig(C.sizeof(T.AedAttnConfig), 8, 8, 128, 1, 1, 32, 128, 0, 1, 0.0)
    for n, v in over.items():
        setattr(c, n, v)
    return c


def attn_bytes(lib, c, q, k, starts=None):
    n = C.c_size_t(0)
    q, pq = T._lens(q)
    k, pk = T._lens(k)
    ps = None
    if starts is not None:
        starts = np.asarray(starts, dtype=np.int64)
        ps = starts.ctypes.data_as(C.POINTER(C.c_int64))
    return lib.aed_attn_workspace_bytes(C.byref(c), pq, pk, ps, len(q), C.byref(n)), n.value


@pytest.mark.parametrize("over,status", [
    (dict(struct_size=4), E), (dict(n_heads=0), E), (dict(n_kv_heads=3), E), (dict(n_kv_heads=0), E), (dict(dtype=2), E), (dict(causal=2), E),
    (dict(training=-1), E), (dict(scale=-1.0), E), (dict(scale=float("nan")), E), (dict(scale=float("inf")), E), (dict(bias_buckets=-1), E),
    (dict(bias_buckets=1), E), (dict(bias_buckets=33, bias_bidirectional=1), E), (dict(bias_buckets=2, bias_bidirectional=1), E),
    (dict(bias_max_distance=16), E), (dict(head_dim=96), U), (dict(bias_buckets=300, bias_max_distance=1000), U), (dict(bias_max_distance=1025), U),
])
def test_attention_configs_are_refused(lib, over, status):
    assert attn_bytes(lib, config(**over), [3, 4], [5, 6])[0] == status
    assert len(lib.aed_train_last_error()) > 10


def test_attention_lengths_are_refused(lib):
    c = config()
    assert attn_bytes(lib, c, [3, -1], [5, 6])[0] == E
    assert attn_bytes(lib, c, [3, 4], [-5, 6])[0] == E
    assert attn_bytes(lib, c, [3, 4], [5, 6], starts=[0, 5])[0] == E        # training needs packed keys
    assert attn_bytes(lib, config(training=0), [3, 4], [5, 6], starts=[0, -5])[0] == E
    assert attn_bytes(lib, c, [3, 4], [5, (1 << 30) + 1])[0] == U
    assert attn_bytes(lib, c, [1 << 30] * 3, [5, 6, 7])[0] == U              # more than 2^31 - 1 rows
    n = C.c_size_t(0)
    one = (C.c_int32 * 1)(4)
    assert lib.aed_attn_workspace_bytes(C.byref(c), one, one, None, 0, C.byref(n)) == E
    assert lib.aed_attn_workspace_bytes(None, one, one, None, 1, C.byref(n)) == E
    assert lib.aed_attn_workspace_bytes(C.byref(c), None, one, None, 1, C.byref(n)) == E
    assert lib.aed_attn_workspace_bytes(C.byref(c), one, one, None, 1, None) == E


def test_attention_workspace(lib):
    status, few = attn_bytes(lib, config(training=0, bias_buckets=0), [1] * 64, [120] * 64)
    assert status == 0 and few < 64 << 10                                    # lists only
    status, n = attn_bytes(lib, config(), [132] * 64, [132] * 64)
    assert status == 0 and 64 * 132 * 8 * 4 + 128 * 8 * 32 * 4 < n < (2 << 20)  # delta, bias sums, lists
    status, n = attn_bytes(lib, config(training=0, bias_buckets=0), [448], [8000])
    assert status == 0 and n > 8 * 448 * 128 * 4 * 2                          # parts of split keys
    # a length of zero is a length
    assert attn_bytes(lib, config(), [0, 5, 0], [4, 0, 0])[0] == 0


def test_create_refuses_before_the_device(lib):
    c, one = config(), (C.c_int32 * 1)(4)
    h = C.c_void_p(None)
    status, n = attn_bytes(lib, c, [4], [4])
    for ws, size in ((None, n), (128, n), (256, n - 1)):
        assert lib.aed_attn_create(C.byref(c), one, one, None, 1, C.c_void_p(ws), size, None, C.byref(h)) == E and not h.value
    assert lib.aed_attn_create(C.byref(c), one, one, None, 1, C.c_void_p(256), n, None, None) == E
    p = T.AedPreferenceConfig(C.sizeof(T.AedPreferenceConfig), 100, 1, 0.1, 0.0)
    two = (C.c_int32 * 2)(4, 5)
    assert lib.aed_preference_create(C.byref(p), two, 1, None, 1 << 20, None, C.byref(h)) == E and not h.value
    # NULL handles
    assert lib.aed_attn_destroy(None) == 0 and lib.aed_preference_destroy(None) == 0
    rows = T.AedRows()
    assert lib.aed_attn_forward(None, rows, rows, rows, None, None, rows, None) == E
    assert lib.aed_attn_backward(None, rows, rows, rows, rows, rows, None, None, None, rows, rows, rows, None) == E
    assert lib.aed_preference_forward(None, None, 1, None, None, None, None, None) == E
    assert lib.aed_preference_backward(None, None, 1, None, None, None, None, None, 1) == E


@pytest.mark.parametrize("over,lens,status", [
    (dict(struct_size=1), [1, 2], E), (dict(vocab=0), [1, 2], E), (dict(dtype=3), [1, 2], E), (dict(beta=0.0), [1, 2], E),
    (dict(beta=float("nan")), [1, 2], E), (dict(label_smoothing=0.5), [1, 2], E), (dict(label_smoothing=-0.1), [1, 2], E), ({}, [1, -2], E),
    ({}, [(1 << 31) - 1, (1 << 31) - 1], U), ({}, [0, 0], 0), (dict(vocab=1), [1, 2], 0),
])
def test_preference_configs(lib, over, lens, status):
    c = T.AedPreferenceConfig(C.sizeof(T.AedPreferenceConfig), 4096, 1, 0.1, 0.0)
    for n, v in over.items():
        setattr(c, n, v)
    lens, p = T._lens(lens)
    n = C.c_size_t(0)
    assert lib.aed_preference_workspace_bytes(C.byref(c), p, len(lens) // 2, C.byref(n)) == status
    assert lib.aed_preference_workspace_bytes(C.byref(c), p, 0, C.byref(n)) == E


def test_work_lists_and_buckets(tmp_path):
    exe = str(tmp_path / "attn_plan")
    r = subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "paper_2503_05931_amd", "csrc"), os.path.join(ROOT, "tests", "native", "attn_plan.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]


def test_reference_buckets():
    """The reference's rule against the table of 32 buckets up to 128, whose edges are known."""
    edges = [n for n in range(1, 130) if R.bucket(n, 32, 128, False) != R.bucket(n - 1, 32, 128, False)]
    assert edges == list(range(1, 17)) + [19, 21, 24, 27, 31, 35, 40, 46, 52, 59, 67, 77, 87, 99, 113]
    assert R.bucket(-5, 32, 128, False) == 0 and R.bucket(-5, 32, 128, True) == 21 and R.bucket(10 ** 6, 32, 128, True) == 15
