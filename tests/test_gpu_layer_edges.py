"""Calls of the layers next to the projection where they can go wrong: values, sizes and lists at the borders of what
their kernels take.  Tolerances are sums of roundings, as in test_gpu_layers.py."""
import math

import pytest

from tests.test_gpu_layers import LEAST, U, _bits, _gen, _half_step, _randn, _same_selection, _select, _t, _torch, _within

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


# ---------------------------------------------------------------- norm
@pytest.mark.parametrize("kind", ["bfloat16", "float32"])
@pytest.mark.parametrize("size", [1e-16, 1e-13, 3e11, 1e14, 1e17])
@pytest.mark.parametrize("d", [96, 1500])
def test_add_norm_grad_of_rows_of_any_size(kind, size, d):
    """Rows so small or so large that rstd^3 is no number of 32 bits any more, though rstd is."""
    torch = _torch()
    import paper_2208_06874_amd as P
    n = 37
    g = _gen(d)
    s, dn = _randn(g, (n, d), kind, size), _randn(g, (n, d), kind)
    w = (1 + _randn(g, (d,), "float32", 0.1)).to(_t(kind))
    r = torch.rsqrt(s.double().square().mean(1)).float()      # (eps = 0)
    dx, dw = P.vp_add_norm_grad(dn, s, w, r)
    rd = r.double()[:, None]
    h, wdy = s.double() * rd, dn.double() * w.double()
    want = rd * (wdy - h * (wdy * h).mean(1, keepdim=True))
    chain = 8 + 6 + -(-d // 512)       # a lane's eight products, six joins of the lanes, the wavefronts
    bound = U * rd * (4 * wdy.abs() + h.abs() * (wdy * h).abs().mean(1, keepdim=True) * (chain + 8))
    _within(dx, want, bound + (want.abs() + bound) * _half_step(kind) + LEAST[kind])
    # one product rounds h, one the term; rows of a wavefront, and its joins, one by one at most
    _within(dw, (dn.double() * h).sum(0), (dn.double() * h).abs().sum(0) * (n + 2) * U)


@pytest.mark.parametrize("n,d", [(1, 64), (5, 64), (7, 600), (2, 2000), (4101, 200)])
def test_add_norm_grad_infinity_in_the_last_row(n, d):
    """Rows are taken four or two at a time: those past the last one count nothing, whatever the last one holds."""
    torch = _torch()
    import paper_2208_06874_amd as P
    s, dn = torch.ones((n, d), device="cuda"), torch.ones((n, d), device="cuda")
    dn[n - 1, 3] = math.inf
    dn[n - 1, d - 1] = -math.inf
    dx, dw = P.vp_add_norm_grad(dn, s, torch.ones(d, device="cuda"), torch.ones(n, device="cuda"))
    want = torch.full((d,), float(n), device="cuda")
    want[3], want[d - 1] = math.inf, -math.inf
    assert torch.equal(dw, want)
    assert torch.isfinite(dx[:n - 1]).all() and dx[n - 1].isnan().all()      # (inf - inf is in the last row's mean)


@pytest.mark.parametrize("d", [1, 65, 300, 513, 2500, 4095])
def test_add_norm_pads_with_zeros_whatever_the_row_holds(d):
    """Columns past d of a row with NaN or infinities, and of one so small that rstd is infinite (eps = 0), are zeros and
    take no part in the last block's scale."""
    torch = _torch()
    import paper_2208_06874_amd as P
    x = torch.ones((4, d), device="cuda")
    x[1, d // 2] = math.nan
    x[2, d // 2] = math.inf
    x[3] = 1e-30                            # (its square is no number above zero: rstd is infinite, and so is y)
    got = P.vp_add_norm(x, torch.ones(d, device="cuda"), eps=0.0, quantize=True, norm_dtype=torch.float32)
    width = -(-d // 128) * 128
    rows = got.q.as_strided((4, width), (width, 1)).view(torch.uint8)
    assert not rows[:, d:].any()
    assert got.norm[3].isinf().all() and got.scales[3].isinf().all() and got.scales[1].isnan().all()
    assert torch.equal(got.scales[0], torch.full_like(got.scales[0], 1.0 / 448))


# ---------------------------------------------------------------- reordering
@pytest.mark.parametrize("bad", [8, 12, 17])
def test_beam_reorder_moves_all_or_nothing(bad):
    """More states than one call of the library takes, one of them refused: the others stay as they are."""
    torch = _torch()
    import paper_2208_06874_amd as P
    parent = torch.tensor([1, 1, 0, 2, 0, 0], dtype=torch.int32, device="cuda")
    states = [(torch.arange(6.0, device="cuda")[:, None] + torch.arange(5.0, device="cuda") * 10 + i, 0) for i in range(18)]
    kept = [t.clone() for t, _ in states]
    wrong = list(states)
    wrong[bad] = (torch.zeros((6, 1), device="cuda").expand(6, 4), 0)
    with pytest.raises(P.VpError, match="overlaps"):
        P.vp_beam_reorder(wrong, parent, 3)
    assert all(torch.equal(t, k) for (t, _), k in zip(states, kept))
    P.vp_beam_reorder(states, parent, 3)
    at = torch.tensor([1, 1, 0, 5, 3, 3], device="cuda")
    assert all(torch.equal(t, k[at]) for (t, _), k in zip(states, kept))
