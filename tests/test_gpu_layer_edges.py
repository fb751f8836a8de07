"""Calls of the layers next to the projection where they can go wrong: values, sizes and lists at the borders of what
their kernels take.  Tolerances are sums of roundings, as in test_gpu_layers.py."""
import math

import pytest

from tests.test_gpu_layers import LEAST, U, _bits, _gen, _half_step, _lists, _quantized, _randn, _same_selection, _select, _t, _torch, _within

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


# ---------------------------------------------------------------- more rows than the threads of one launch
def _room(gigabytes):
    """Skips where the card has not this much memory free."""
    torch = _torch()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes * 1.2e9:
        pytest.skip("needs %d GB of GPU memory" % gigabytes)


@pytest.mark.parametrize("n,d", [(2 ** 30 + 77, 1), (2 ** 24 + 3, 520)])
def test_embed_of_more_rows_than_a_launch_has_threads(n, d):
    """Four threads a row at least and 256 at most: 2^32 threads and more, and what lies on both sides of where launches meet."""
    torch = _torch()
    import paper_2208_06874_amd as P
    _room(50)
    V = 1000
    t = _randn(_gen(d), (V, d), "float32")
    ids = torch.arange(n, device="cuda", dtype=torch.int32) % V
    ids[5::1 << 20] = -1
    got = P.vp_embed(t, ids)
    at = torch.cat([torch.arange(s, min(s + 2000, n), device="cuda") for s in (0, 2 ** 23 - 1000, 2 ** 24 - 1000, 2 ** 29 - 1000, 2 ** 30 - 1000, n - 2000) if s < n])
    want = torch.where(ids[at, None] >= 0, t[ids[at].long().clamp(min=0)], 0.0)
    assert torch.equal(got[at], want)
    step = max(1, 2 ** 26 // d)
    for a in range(0, n, step):              # every row was written
        i = ids[a:a + step].long()
        assert torch.equal(got[a:a + step, 0], torch.where(i >= 0, t[i.clamp(min=0), 0], 0.0)), a


@pytest.mark.parametrize("n,d", [(2 ** 26 + 5, 8), (2 ** 25 + 3, 520)])
def test_add_norm_of_more_rows_than_a_launch_has_threads(n, d):
    """64 threads a row, and 128.  The rows are a few, over and over: equal rows give equal results."""
    torch = _torch()
    import paper_2208_06874_amd as P
    _room(20 + 7 * n * d / 1e9)      # (four of 16 bits, rows of q at multiples of 128 bytes)
    few = 61
    g = _gen(d)
    rows, rest, w = _randn(g, (few, d), "bfloat16"), _randn(g, (few, d), "bfloat16"), _randn(g, (d,), "float32")
    x, r = rows.repeat(-(-n // few), 1)[:n], rest.repeat(-(-n // few), 1)[:n]
    want = P.vp_add_norm(rows, w, residual=rest, norm_dtype=torch.bfloat16, quantize=True, rstd=True)
    got = P.vp_add_norm(x, w, residual=r, norm_dtype=torch.bfloat16, quantize=True, rstd=True, inplace=True)
    assert got.sum is r
    step = few * (2 ** 24 // d + 1)
    for a in range(0, n, step):
        for name in ("sum", "norm", "q", "scales", "rstd"):
            here, base = getattr(got, name)[a:a + step], getattr(want, name)
            if name == "q":
                here, base = here.view(torch.uint8), base.view(torch.uint8)
            whole = here.shape[0] // few * few
            assert (here[:whole].view(-1, *base.shape) == base).all() if here.is_contiguous() else (here[:whole].unflatten(0, (-1, few)) == base).all(), (name, a)
            assert torch.equal(here[whole:], base[:here.shape[0] - whole]), (name, a)


@pytest.mark.parametrize("n,V", [(3000, 2 ** 28 + 21), (700, 2 ** 31 - 17)])
def test_embed_grad_of_more_tokens_than_a_launch_has_threads(n, V):
    """Through lists (16 threads a token) and without (two); tokens on both sides of where launches meet, and the last ones."""
    torch = _torch()
    import paper_2208_06874_amd as P
    _room(30)
    g = _gen(n)
    edges = [t for t in (0, 2 ** 27, 2 ** 28, 2 ** 30) if t < V] + [V]
    near = torch.cat([torch.arange(max(0, t - 20), min(t + 20, V), device="cuda") for t in edges])
    ids = near[torch.randint(0, len(near), (n,), generator=g, device="cuda")].to(torch.int32)
    ids[::7] = int(near[30])                              # (a list that is cut into windows)
    x = torch.randint(-8, 9, (n, 1), generator=g, device="cuda").half()      # (sums of whole numbers are exact)
    grad = torch.full((V, 1), math.nan, dtype=torch.float16, device="cuda")
    P.vp_embed_grad(x, ids, V, out=grad)
    at, slot = torch.unique(ids.long(), return_inverse=True)
    want = torch.zeros((len(at), 1), device="cuda").index_add_(0, slot, x.float())
    assert torch.equal(grad[at].float(), want)
    grad[at] = 0
    for a in range(0, V, 2 ** 28):
        assert not grad[a:a + 2 ** 28].view(torch.int16).any(), a


def test_beam_reorder_of_more_pieces_than_a_launch_has_threads():
    """Bytes whose rows are innermost: a thread for each place of every sentence, in three states one behind the other."""
    torch = _torch()
    import paper_2208_06874_amd as P
    _room(25)
    S, B = 4, 2
    n = S * B
    parent = torch.tensor([1, 0, 0, 0, 1, 1, -1, 0], dtype=torch.int32, device="cuda")
    at = torch.tensor([1, 0, 2, 2, 5, 5, 6, 6], device="cuda")
    step = 2 ** 26
    line = (torch.arange(step * n, device="cuda") * 7 >> 1).to(torch.uint8).view(step, n)      # (a byte for each place and row)
    states = [line.repeat(k, 1) for k in (3, 13, 1)]
    assert sum(t.numel() // B for t in states) > 2 ** 32
    P.vp_beam_reorder([(t, 1) for t in states], parent, B)
    want = line[:, at]
    for t in states:
        for a in range(0, t.shape[0], step):
            assert torch.equal(t[a:a + step], want), a


def test_scaled_pack_of_more_pieces_than_a_launch_has_threads():
    """64 GiB and more of weights, a thread for every 16 bytes: the product with rows on both sides of where launches meet."""
    torch = _torch()
    import paper_2208_06874_amd as P
    M, d = 2 ** 22 + 200, 16384
    _room(2 * M * d / 1e9)
    wq = torch.zeros((M, d), dtype=torch.uint8, device="cuda")
    at = torch.tensor([0, 31, M // 2 - 150, M // 2, 2 ** 21 - 1, 2 ** 21, 2 ** 21 + 77, 2 ** 22 - 1, 2 ** 22, M - 33, M - 1], device="cuda")
    g = _gen(7)
    rows = torch.randint(-8, 9, (len(at), d), generator=g, device="cuda").float()
    wq[at] = rows.to(torch.float8_e4m3fn).view(torch.uint8)
    packed = P.vp_scaled_pack(wq.view(torch.float8_e4m3fn), torch.ones((-(-M // 128), d // 128), device="cuda"))
    x = torch.randint(-8, 9, (3, d), generator=g, device="cuda").float()
    z = P.vp_scaled_matmul(packed, x.to(torch.float8_e4m3fn), torch.ones((3, d // 128), device="cuda"), out_dtype=torch.float32)
    assert torch.equal(z[:, at].double(), x.double() @ rows.double().t().contiguous())      # (whole numbers: exact)
    z[:, at] = 0
    assert not z.any()


# ---------------------------------------------------------------- lists of the embedding's gradient
def _clustered(n, V, where):
    """Tokens from 20 on all over, none of them often; `where`: token -> the positions that it has."""
    torch = _torch()
    ids = 20 + (torch.arange(n, device="cuda") * 7919 % (V - 20)).to(torch.int32)
    for token, at in where.items():
        ids[at] = token
    return ids


@pytest.mark.parametrize("kind", ["lengths", "a run in a wide window", "a run in narrow windows", "a long run in a wide window", "every second", "two tokens"])
@pytest.mark.parametrize("d,dout,grad", [(24, "float16", "float32"), (520, "bfloat16", "bfloat16"), (1031, "float32", "float32")])
def test_embed_grad_lists(kind, d, dout, grad):
    """Lists whose positions are found and ordered in each of the ways there are."""
    torch = _torch()
    import paper_2208_06874_amd as P
    r = lambda a, b, s=1: torch.arange(a, b, s, device="cuda")  # noqa: E731
    n, V, where = {
        # at the borders of one wavefront's lists, of one window, of two
        "lengths": (9000, 4000, {k: r(100 * k, 100 * k + 99 * (c - 1) + 1, 99) % 9000 if c < 90 else r(5000 + k, 5000 + k + 13 * c, 13) % 9000
                                 for k, c in enumerate((1, 15, 16, 17, 127, 128, 129, 256, 257))}),
        # 300 positions, cut into three windows of 13,334, all in one: more than are ordered by comparing, twice 8,192 positions as bits
        "a run in a wide window": (40000, 30000, {3: r(20000, 20300)}),
        # 10,000 in 79 windows of 2,532 positions: fewer than the list has entries
        "a run in narrow windows": (200000, 30000, {3: r(50000, 60000)}),
        # 9,000 in 71 windows of 14,085, nearly all in two of them
        "a long run in a wide window": (1000000, 30000, {3: r(500000, 509000)}),
        "every second": (30000, 5000, {1: r(0, 30000, 2)}),
        "two tokens": (20001, 30, {0: r(0, 20001), 5: r(3, 20001, 17)})}[kind]
    if kind == "a long run in a wide window" and d > 600:
        n, where = 600000, {3: r(300000, 309000)}
    ids = _clustered(n, V, where)
    x = _randn(_gen(d), (n, d), dout)
    got = P.vp_embed_grad(x, ids, V, scale=0.5, grad_dtype=_t(grad))
    at = ids.long()
    count = torch.bincount(at, minlength=V).double()
    assert kind != "lengths" or count[:9].tolist() == [1, 15, 16, 17, 127, 128, 129, 256, 257]
    want, size = (torch.zeros((V, d), dtype=torch.float64, device="cuda") for _ in range(2))
    for a in range(0, n, 100000):
        want.index_add_(0, at[a:a + 100000], x[a:a + 100000].double() * 0.5)
        size.index_add_(0, at[a:a + 100000], x[a:a + 100000].double().abs() * 0.5)
    _within(got, want, size * (count[:, None] + 1) * U + want.abs() * _half_step(grad) * 1.001 + LEAST[grad])
    assert torch.equal(got, P.vp_embed_grad(x, ids, V, scale=0.5, grad_dtype=_t(grad)))


def test_embed_grad_of_one_token_goes_with_its_positions():
    """Four times the positions of one token take about four times as long, not sixteen."""
    torch = _torch()
    import paper_2208_06874_amd as P

    def least(n):
        ids, x, best = torch.full((n,), 7, device="cuda", dtype=torch.int32), torch.ones((n, 4), device="cuda", dtype=torch.float16), math.inf
        out = P.vp_embed_grad(x, ids, 100)
        assert float(out[7, 0]) == n and float(out.sum()) == 4 * n      # (whole numbers below 2^24: exact)
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            P.vp_embed_grad(x, ids, 100)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    few, many = least(2 ** 20), least(2 ** 22)
    assert many < 9 * few, "%.3f and %.3f ms" % (few, many)


# ---------------------------------------------------------------- 8-bit product
def _cut(xq, wq):
    """What the 8-bit matrix instructions may lose: 7 * 2^-13 of the largest product's binade of every eight columns [n, M, d / 8]
    -> by column blocks [d / 128, n, M] (subnormal values at the exponent that they have)."""
    torch = _torch()
    power = lambda q: torch.where(q == 0, torch.zeros((), device="cuda"), torch.exp2(torch.floor(torch.log2(q.float().abs().clamp(min=2.0 ** -6)))))  # noqa: E731
    d = xq.shape[1]
    ex, ew, out = power(xq), power(wq), []
    for b in range(0, d, 128):
        lost = torch.zeros((xq.shape[0], wq.shape[0]), device="cuda")
        for g in range(b, b + 128, 8):
            most = torch.zeros_like(lost)
            for k in range(g, min(g + 8, d)):
                most = torch.maximum(most, ex[:, k, None] * ew[None, :, k])
            lost += most
        out.append(lost * 7 * 2.0 ** -13)
    return torch.stack(out)


@pytest.mark.parametrize("n,M,d", [(1, 3000, 640), (16, 700, 1024), (33, 900, 384), (300, 1100, 512), (128, 131072, 256)])
@pytest.mark.parametrize("kind", ["one column", "one of eight, one sign", "all sizes"])
@pytest.mark.parametrize("out", ["float16", "bfloat16", "float32"])
def test_scaled_matmul_of_columns_of_different_sizes(n, M, d, kind, out):
    """Columns far larger than the others, as the output of a norm has them: 16-bit outputs lose no more than documented, fp32
    outputs nothing."""
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(n + M)
    x, w = torch.randn((n, d), generator=g, device="cuda"), torch.randn((M, d), generator=g, device="cuda")
    if kind == "one column":
        x[:, 77::128] *= 200
    elif kind == "all sizes":
        x, w = x * torch.exp2(4 * torch.randn((n, d), generator=g, device="cuda")), w * torch.exp2(2 * torch.randn((M, d), generator=g, device="cuda"))
    else:
        x, w = x.abs(), w.abs()
        x[:, ::8] *= 2000
    (xq, xs), (wq, ws) = _quantized(x, 1), _quantized(w, 128)
    got = P.vp_scaled_matmul(P.vp_scaled_pack(wq, ws), xq, xs, out_dtype=_t(out))
    of = torch.arange(M, device="cuda") // 128
    X = xq.float().double() * xs.double().repeat_interleave(128, 1)[:, :d]
    W = (wq.float().double() * ws.double()[of].repeat_interleave(128, 1)[:, :d]).t().contiguous()
    lost = torch.zeros((n, M), dtype=torch.float64, device="cuda")
    if out != "float32":
        for b, cut in enumerate(_cut(xq, wq)):
            lost += cut.double() * xs.double()[:, b, None] * ws.double()[of, b][None]
    for a in range(0, M, 4096):
        want, size = X @ W[:, a:a + 4096].contiguous(), X.abs() @ W[:, a:a + 4096].abs().contiguous()
        # within a block 128 additions that may cut off rather than round (2^-23 each); then the blocks and the scales
        bound = size * (128 * 2 * U + (-(-d // 128) + 4) * U) + lost[:, a:a + 4096]
        bound += (want.abs() + bound) * _half_step(out) + LEAST[out]
        z, most = got[:, a:a + 4096].double(), torch.finfo(_t(out)).max
        past = z.isinf() & (z * want > 0) & (want.abs() + bound > most)         # (what is past the type's range becomes infinite)
        assert past.all() or not (want.abs() - bound > most * (1 + _half_step(out)))[~past].any()
        _within(torch.where(past, want, z), want, bound)


# ---------------------------------------------------------------- graphs, streams, long offsets on the paths of many rows
def test_embed_grad_through_lists_replayed_from_a_graph():
    """More than 1,024 positions: counters, cursors and lists in the workspace are cleared by every replay."""
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(31)
    n, V, d = 9000, 700, 130
    x, ids = _randn(g, (n, d), "bfloat16"), _lists("mixed", n, V, g)
    P.vp_embed_grad(x, ids, V, padding_id=1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = P.vp_embed_grad(x, ids, V, padding_id=1)
    for rep in range(6):
        ids.copy_(_lists(("mixed", "one", "few", "runs")[rep % 4], n, V, g))
        x.copy_(_randn(g, (n, d), "bfloat16"))
        want = P.vp_embed_grad(x, ids, V, padding_id=1).clone()
        torch.cuda.synchronize()
        print("replay", rep, flush=True)
        held.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want)


@pytest.mark.parametrize("n,M,d,out", [(600, 4000, 300, "float16"), (600, 4000, 300, "float32"), (130, 70000, 256, "bfloat16"), (40, 5000, 700, "float16")])
def test_scaled_matmul_of_many_rows_replayed_from_a_graph(n, M, d, out):
    """The rows are laid out in the workspace first."""
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(n)
    (xq, xs), (wq, ws) = _quantized(_randn(g, (n, d), "float32"), 1), _quantized(_randn(g, (M, d), "float32"), 128)
    packed, b = P.vp_scaled_pack(wq, ws), _randn(g, (M,), "float32")
    P.vp_scaled_matmul(packed, xq, xs, bias=b, out_dtype=_t(out))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = P.vp_scaled_matmul(packed, xq, xs, bias=b, out_dtype=_t(out))
    for rep in range(4):
        q, s = _quantized(_randn(g, (n, d), "float32"), 1)
        xq.copy_(q), xs.copy_(s)
        want = P.vp_scaled_matmul(packed, xq, xs, bias=b, out_dtype=_t(out)).clone()
        torch.cuda.synchronize()
        print("replay", rep, flush=True)
        held.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want)


def test_selection_of_many_rows_replayed_from_a_graph():
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(33)
    S, B, V = 24, 8, 30011
    n = S * B
    z, scores = _randn(g, (n, V), "float16", 2.0), -torch.rand(n, generator=g, device="cuda")
    bits, done = _bits(g, n, V, 0.8), (torch.rand(n, generator=g, device="cuda") < 0.2).to(torch.uint8)
    f = lambda: P.vp_beam_select(z, scores, B, allowed=bits, done=done, eos=2)  # noqa: E731
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = f()
    for rep in range(4):
        z.copy_(torch.zeros_like(z) if rep == 2 else _randn(g, (n, V), "float16", 2.0))      # (ties of whole rows once)
        scores.copy_(-torch.rand(n, generator=g, device="cuda"))
        want = [t.clone() for t in f()]
        torch.cuda.synchronize()
        print("replay", rep, flush=True)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_paths_of_many_rows_on_other_streams():
    """Lists of the embedding's gradient and rows of the product, each call with a workspace on its own stream, interleaved."""
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(34)
    n, V, d, M = 9000, 900, 200, 3000
    x, ids = _randn(g, (n, d), "float16"), _lists("mixed", n, V, g)
    (xq, xs), (wq, ws) = _quantized(_randn(g, (n, d), "float32"), 1), _quantized(_randn(g, (M, d), "float32"), 128)
    packed = P.vp_scaled_pack(wq, ws)
    want = P.vp_embed_grad(x, ids, V), P.vp_scaled_matmul(packed, xq, xs)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for rep in range(9):
        st = streams[rep % 3]
        if rep % 2:
            got.append((P.vp_embed_grad(x, ids, V, stream=st), P.vp_scaled_matmul(packed, xq, xs, stream=st)))
        else:
            with torch.cuda.stream(st):
                got.append((P.vp_embed_grad(x, ids, V), P.vp_scaled_matmul(packed, xq, xs)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[0]) and torch.equal(b, want[1]) for a, b in got)


def test_embed_grad_through_lists_past_32_bits():
    """Rows of the gradient, and of what it is made of, past 2^31 elements."""
    torch = _torch()
    import paper_2208_06874_amd as P
    _room(16)
    d, V, n = 4096, 600000, 530000
    tokens = torch.tensor([0, V - 1, V // 2, 524287, 524288, 524289], dtype=torch.int32, device="cuda")
    ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, n - 1, 524288, 524287, 7, 524290], device="cuda")
    ids[at] = tokens
    ids[n - 500:n - 1] = V - 1                            # (a list of several windows)
    x = torch.zeros((n, d), dtype=torch.float16, device="cuda")
    rows = torch.randint(-8, 9, (6, d), generator=_gen(1), device="cuda").half()
    x[at] = rows
    x[n - 500:n - 1, ::3] = 1.0
    grad = torch.full((V, d), math.nan, dtype=torch.float16, device="cuda")
    P.vp_embed_grad(x, ids, V, out=grad)
    want = rows.clone()
    want[1, ::3] += 499
    assert torch.equal(grad[tokens.long()], want)
    grad[tokens.long()] = 0
    assert not grad.view(torch.int16).any()


def test_logits_past_32_bits_to_their_own_rounding():
    """fp32 logits are sums in 32 bits: no more than those roundings, past 2^31 elements."""
    torch = _torch()
    import paper_2208_06874_amd as P
    _room(12)
    n, M, d = 2000, 1200000, 32
    g = _gen(2)
    (xq, xs), (wq, ws) = _quantized(_randn(g, (n, d), "float32"), 1), _quantized(_randn(g, (M, d), "float32"), 128)
    z = P.vp_scaled_matmul(P.vp_scaled_pack(wq, ws), xq, xs, out_dtype=torch.float32)
    at = torch.tensor([0, 1, 999, 1789, 1790, 1999], device="cuda")
    x = xq[at].float().double() * xs[at].double()
    w = (wq.float().double() * ws.double().repeat_interleave(128, 0)[:M]).t().contiguous()
    want = x @ w
    _within(z[at], want, (x.abs() @ w.abs()) * (32 * 2 + 5) * U + want.abs() * U)       # 32 additions that may cut off, the scales


# ---------------------------------------------------------------- norm, to the sums as they are made
@pytest.mark.parametrize("n,d,kind", [(300, 500, "float32"), (300, 512, "bfloat16"), (200, 1024, "float32"), (200, 1500, "float32"), (100, 2049, "float16"), (100, 4096, "float32"), (7, 3600, "bfloat16")])
def test_add_norm_to_its_own_roundings(n, d, kind):
    """A lane adds eight squares, six joins the lanes of a wavefront, and the row's wavefronts follow one by one."""
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(n + d)
    x, r, w = _randn(g, (n, d), kind), _randn(g, (n, d), kind), (1 + _randn(g, (d,), "float32", 0.1))
    eps = float(torch.tensor(1e-6))
    got = P.vp_add_norm(x, w, residual=r, eps=eps, norm_dtype=torch.float32, rstd=True)
    s = (x.float() + r.float()).to(x.dtype)
    assert torch.equal(got.sum, s)
    f = s.double()
    rstd = 1 / torch.sqrt(f.square().mean(1) + eps)
    rel = ((8 + 6 + -(-d // 512) - 1) / 2 + 4) * U       # (the root halves; mean, eps, root, quotient)
    _within(got.rstd, rstd, rstd * rel)
    y = f * rstd[:, None] * w.double()
    _within(got.norm, y, y.abs() * (rel + 2 * U))


@pytest.mark.parametrize("n,d", [(3, 100), (4097, 500), (9000, 512), (5000, 1000), (2100, 1024), (5000, 1500), (1025, 4096), (3100, 2050)])
def test_add_norm_grad_of_the_weight_to_its_own_roundings(n, d):
    """Up to 1,024 workgroups of four, two or one rows (rows of up to 512, of up to 1,024, wider): the rows of a wavefront, the rows of
    a workgroup, the workgroups in 32 strands, and five joins of these."""
    torch = _torch()
    import paper_2208_06874_amd as P
    g = _gen(n + d)
    s, dn, w = _randn(g, (n, d), "float32", 3.0), _randn(g, (n, d), "float32"), _randn(g, (d,), "float32")
    r = torch.rsqrt(s.double().square().mean(1) + 1e-6).float()
    _, dw = P.vp_add_norm_grad(dn, s, w, r)
    together = 4 if d <= 512 else 2 if d <= 1024 else 1
    groups = min(1024, -(-n // together))
    chain = -(-n // (groups * together)) + (together - 1) + -(-groups // 32) + 5 + 1      # (and the rounding of s * rstd)
    terms = dn.double() * s.double() * r.double()[:, None]
    _within(dw, terms.sum(0), terms.abs().sum(0) * chain * U)
