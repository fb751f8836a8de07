"""Calls of the layers next to the projection where they can go wrong: values, sizes and lists at the borders of what
their kernels take.  Tolerances are sums of roundings, as in test_gpu_layers.py."""
import pytest

from tests.test_gpu_layers import _bits, _gen, _randn, _same_selection, _select, _t, _torch

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- selection
@pytest.mark.parametrize("V", [65, 40000])
@pytest.mark.parametrize("kind,patterns", [("float16", (0x7c01, -0x3ff, 0x7dff)), ("bfloat16", (0x7f81, -0x7f, 0x7fbf)),
                                           ("float32", (0x7f800001, -0x7fffff, 0x7fbfffff))])
def test_beam_select_signalling_nan(kind, patterns, V):
    """Signalling NaN (infinity's exponent, a mantissa without its first bit, both signs) count as tokens that are not
    allowed, like quiet ones."""
    torch = _torch()
    import paper_2208_06874_amd as P
    B, S = 4, 2
    n = S * B
    g = _gen(V)
    z = _randn(g, (n, V), kind)
    i = z.view(torch.int32 if kind == "float32" else torch.int16)
    for row, p in enumerate(patterns):
        i[row, 5] = p
    i[3, :64] = patterns[0]                 # whole vectors of them
    i[4, 1:] = patterns[1]                  # all but one token
    i[5, ::2] = patterns[2]
    i[6] = patterns[0]                      # nothing else
    assert z.isnan()[[0, 1, 2, 3, 4, 5, 6], [5, 5, 5, 0, 1, 0, 0]].all()
    scores = -torch.rand(n, generator=g, device="cuda")
    for allowed in (None, _bits(g, n, V, 0.7)):
        _same_selection(P.vp_beam_select(z, scores, B, allowed=allowed), _select(z, scores, B, allowed))
