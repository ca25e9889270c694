"""Which scales attention's validation lets through, seen from the refusal that comes next: no case passes validation, so
nothing is launched and no GPU is needed."""
from helpers import load_binding

b = load_binding()

from test_abi_host_attention import INVALID, WS, bwd, fwd  # noqa: E402


def test_scales():
    """2^-100 to 2^100: past the ends lse / scale, or scale in base 2, could pass the largest float."""
    for call in (fwd, bwd):
        for bad in (2.0 ** -101, 1e-37, 1e-40, 2.0 ** 101, 3e38):
            assert call(scale=bad) == INVALID
    for good in (2.0 ** -100, 0.125, 1.0, 2.0 ** 100):
        assert bwd(scale=good, ws=None, ws_bytes=0) == WS
