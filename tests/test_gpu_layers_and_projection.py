"""The layers next to the projection with the projection itself: a decode loop in which the embedding's and the norm's rows are
what vp_project takes, and vp_beam_step's parents and tokens are what moves the states and is embedded next."""
import math

import numpy as np
import pytest

from paper_2208_06874_amd import workloads as wl
from tests import parity_util as pu
from tests.test_gpu_layers import LEAST, U, _half_step, _moved, _torch, _within
from tests.test_gpu_search import _dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,B", [(4, 4), (1, 5)])
def test_decode_loop(oracle, S, B):
    torch = _torch()
    import paper_2208_06874_amd as P
    cfg = wl.CONFIGS["tiny"]
    W, b, C = wl.make_model(cfg)
    off, ids = wl.make_candidates(cfg, W, b, C, device="cuda:0")
    index = P.vp_build(_dev(W), _dev(b), _dev(C), off, ids, k_max=8)
    table = _dev(W.T)                       # (one table for both ends)
    n, d, k, steps, eps = S * B, cfg.d, 4, 5, float(np.float32(1e-6))
    weight = torch.ones(d, dtype=torch.float16, device="cuda")
    scores = torch.full((S, B), -math.inf, device="cuda")
    scores[:, 0] = 0
    scores = scores.view(-1)
    token = (10 + torch.arange(S, device="cuda", dtype=torch.int32)).repeat_interleave(B)
    stream = _dev(wl.make_rows(cfg, C, N=n)[0]).clone()
    history = torch.full((n, steps), -1, dtype=torch.int32, device="cuda")
    for step in range(steps):
        before = stream.clone()
        x = P.vp_embed(table, token, scale=math.sqrt(d))
        r = P.vp_add_norm(x, weight, residual=stream, eps=eps, inplace=True)
        assert r.sum is stream and torch.equal(stream, (x.float() + before.float()).half())
        f = stream.double()
        y = f / torch.sqrt(f.square().mean(1, keepdim=True) + eps)
        # eight squares a lane and six joins, half of their relative error; root, quotient, products
        _within(r.norm, y, y.abs() * ((14 / 2 + 6) * U + _half_step("float16")) * 1.001 + LEAST["float16"])
        out_ids, out_logp, g = P.vp_project(index, r.norm, k)
        torch.cuda.synchronize()
        pu.check_projection(oracle, W, b, C, off, ids, pu.to_np(r.norm), k, pu.to_np(out_ids), pu.to_np(out_logp), pu.to_np(g))
        want = oracle.beam_step(pu.to_np(out_ids), pu.to_np(out_logp), pu.to_np(scores), B)
        scores, parent, token = P.vp_beam_step(out_ids, out_logp, scores, B)
        assert all(np.array_equal(pu.to_np(a), w) for a, w in zip((scores, parent, token), want))
        held = [(stream, 0), (history[:, :step], 0)]
        moved = [_moved(t, dim, parent, B) for t, dim in held]
        P.vp_beam_reorder(held, parent, B)
        assert all(torch.equal(t, m) for (t, _), m in zip(held, moved))
        history[:, step] = token
        assert not P.vp_embed(table, token)[token < 0].any()       # (a missing hypothesis has no token)
    assert torch.isfinite(scores).all() and (history >= 0).all()
    assert len({tuple(h) for h in history.tolist()}) == n
