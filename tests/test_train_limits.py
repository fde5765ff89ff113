"""Limits of the training operators that are checked on the host, from both sides.  No GPU work."""
from paper_2503_05931_amd import binding
from tests.test_train_abi import attn_bytes, config, lib  # noqa: F401 (lib: the fixture)


def test_key_starts(lib):  # noqa: F811
    c = config(training=0)
    assert attn_bytes(lib, c, [1, 1], [0, 1], starts=[0, 1 << 38])[0] == 0
    assert attn_bytes(lib, c, [1, 1], [0, 1], starts=[0, (1 << 38) + 1])[0] == binding.AED_EINVAL
    assert attn_bytes(lib, c, [1, 1], [0, 1], starts=[0, (1 << 63) - 1])[0] == binding.AED_EINVAL
