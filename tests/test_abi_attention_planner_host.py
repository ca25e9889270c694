"""How many shares of the keys the forward attention plans, from its workspace answers (no GPU is needed)."""
import ctypes

import pytest

from helpers import load_binding

b = load_binding()

from test_abi_host import BF16, D, F32, R  # noqa: E402


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,TQ,TK,HQ,HK,W", [(4, 1, 8801, 16, 16, 128), (25, 2, 1624, 32, 8, 128), (20, 16, 2346, 32, 8, 64),
                                             (3, 2, 8149, 32, 8, 128), (9, 1, 6326, 32, 8, 128)])
def test_shares_of_the_keys_do_not_depend_on_lengths(dtype, B, TQ, TK, HQ, HK, W):
    """Lengths are on the device and may all be full: the plan is that of a call without them."""
    def need(kv_len):
        n = ctypes.c_size_t()
        t = lambda T, H, at: D([B, T, H, W], dtype, at << 40)
        assert b.lib.mt_attention_fwd_workspace(R(t(TQ, HQ, 1)), R(t(TK, HK, 2)), R(t(TK, HK, 3)), R(kv_len), None,
                                                R(t(TQ, HQ, 4)), None, 0, ctypes.byref(n)) == 0
        return n.value
    assert need(D([B], b.I32, 0xa00000)) == need(None)
