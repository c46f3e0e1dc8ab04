"""The cross entropy's scale on the host: one whose exponents would pass FP32's range is refused."""
import pytest

from test_train_abi import BAD, FAKE, L, WS, XENT, head, packed  # noqa: F401


@pytest.mark.parametrize("scale,code", [(2.0 ** 127, WS), (-2.0 ** 127, WS), (2.0 ** 127 * 1.01, BAD),
                                        (-2.0 ** 127 * 1.01, BAD), (3.4e38, BAD), (1e-45, WS), (0.0, WS)])
def test_scales(L, scale, code):  # noqa: F811
    """(Those that are taken get as far as the missing workspace.)"""
    assert L.embbag_xent(packed(head._Xent, XENT, dict(scale=scale)), None, 0, None, None) == code
