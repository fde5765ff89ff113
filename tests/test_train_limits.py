"""Limits of the training operators that are checked on the host, from both sides.  No GPU work."""
import ctypes as C

import numpy as np

from paper_2503_05931_amd import binding, training as T
from tests.test_train_abi import attn_bytes, config, lib  # noqa: F401 (lib: the fixture)


def test_key_starts(lib):  # noqa: F811
    c = config(training=0)
    assert attn_bytes(lib, c, [1, 1], [0, 1], starts=[0, 1 << 38])[0] == 0
    assert attn_bytes(lib, c, [1, 1], [0, 1], starts=[0, (1 << 38) + 1])[0] == binding.AED_EINVAL
    assert attn_bytes(lib, c, [1, 1], [0, 1], starts=[0, (1 << 63) - 1])[0] == binding.AED_EINVAL


def test_workgroups_of_attention(lib):  # noqa: F811
    """A launch of 256 threads a workgroup has less than 2^32 threads: 2^24 - 1 workgroups, in every list."""
    U, most = binding.AED_EUNSUPPORTED, (1 << 24) - 1
    few = config(training=0, bias_buckets=0, n_heads=16, n_kv_heads=16)
    n = most // 16
    assert attn_bytes(lib, few, np.ones(n, np.int32), np.ones(n, np.int32))[0] == 0                # one row a sequence: an item each
    assert attn_bytes(lib, few, np.ones(n + 1, np.int32), np.ones(n + 1, np.int32))[0] == U
    # query gradients: an item each of 128 rows, where the forward kernel has them too
    many = config(bias_buckets=0, n_heads=4096, n_kv_heads=1)
    rows = most // 4096 * 128
    assert attn_bytes(lib, many, [rows], [64])[0] == 0
    assert attn_bytes(lib, many, [rows + 1], [64])[0] == U
    # key gradients, and behind them the bias's: a workgroup for four sums
    keys = config(bias_buckets=0, n_heads=4096, n_kv_heads=4096)
    assert attn_bytes(lib, keys, [64], [rows])[0] == 0
    assert attn_bytes(lib, keys, [64], [rows + 1])[0] == U
    assert attn_bytes(lib, config(bias_buckets=4, n_heads=4096, n_kv_heads=4096), [64], [rows - 128])[0] == 0    # 4 094 x 4 096 + 4 096
    assert attn_bytes(lib, config(bias_buckets=4, n_heads=4096, n_kv_heads=4096), [64], [rows])[0] == U
    # nothing is built for what is refused: the largest lists
    assert attn_bytes(lib, config(n_heads=65535, n_kv_heads=65535), [1 << 30], [1 << 30])[0] == U


def test_rows_of_the_preference_loss(lib):  # noqa: F811
    """Four rows a workgroup."""
    c = T.AedPreferenceConfig(C.sizeof(T.AedPreferenceConfig), 8, 1, 0.1, 0.0)
    n = C.c_size_t(0)
    for rows, status in (((1 << 26) - 4, 0), ((1 << 26) - 3, binding.AED_EUNSUPPORTED)):
        lens, p = T._lens([rows - 1, 1])
        assert lib.aed_preference_workspace_bytes(C.byref(c), p, 1, C.byref(n)) == status
