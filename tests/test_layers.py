"""CPU-side checks of the layers' entry points: what they refuse, on the host and before anything is launched."""
import ctypes

import pytest
import torch

import paper_2208_06874_amd as P
from paper_2208_06874_amd import layers, vp

OK, INVALID, UNSUPPORTED, WORKSPACE = vp.VP_OK, vp.VP_ERR_INVALID_ARG, vp.VP_ERR_UNSUPPORTED, vp.VP_ERR_WORKSPACE
A = 0x10000     # an address that is never read


def _call(name, **kw):
    """The entry point with arguments that are fine as they stand, but for those in kw."""
    base = dict(
        vp_embed=dict(table=A, table_type=0, stride=64, V=100, d=64, ids=A, n=5, scale=1.0, out=A, out_type=0, stream=None),
        vp_embed_grad=dict(dout=A, dout_type=0, stride=64, ids=A, n=500, V=100, d=64, scale=1.0, pad=-1, grad=A, grad_type=2, ws=A, ws_bytes=1 << 30, stream=None),
        vp_add_norm=dict(x=A, x_stride=64, residual=A, r_stride=64, type=0, weight=A, weight_type=2, n=5, d=64, eps=1e-6, sum=A, norm=A, norm_type=0, q=A,
                         scales=A, rstd=A, stream=None),
        vp_add_norm_grad=dict(dnorm=A, dn_stride=64, s=A, s_stride=64, dsum=A, ds_stride=64, type=0, weight=A, weight_type=0, rstd=A, n=5, d=64, dx=A,
                              dweight=A, ws=A, ws_bytes=1 << 30, stream=None),
        vp_scaled_pack=dict(wq=A, stride=64, ws=A, M=100, d=64, packed=A, packed_bytes=1 << 30, stream=None),
        vp_scaled_matmul=dict(packed=A, M=100, d=64, xq=A, stride=64, xs=A, n=5, bias=A, bias_type=0, out=A, out_type=0, ws=A, ws_bytes=1 << 30, stream=None),
        vp_beam_select=dict(logits=A, type=0, stride=100, scores=A, S=2, B=3, V=100, allowed=A, a_stride=4, done=A, eos=2, out_scores=A, out_parent=A,
                            out_token=A, out_done=A, ws=A, ws_bytes=1 << 30, stream=None),
    )[name]
    assert set(kw) <= set(base)
    return getattr(vp.lib(), name)(*dict(base, **kw).values())


@pytest.mark.parametrize("name,kw,status", [
    ("vp_embed", dict(table=None), INVALID), ("vp_embed", dict(ids=None), INVALID), ("vp_embed", dict(out=None), INVALID),
    ("vp_embed", dict(table_type=3), INVALID), ("vp_embed", dict(out_type=-1), INVALID), ("vp_embed", dict(stride=63), INVALID),
    ("vp_embed", dict(table=A + 1), INVALID), ("vp_embed", dict(table=A + 2, table_type=2), INVALID), ("vp_embed", dict(out=A + 2, out_type=2), INVALID),
    ("vp_embed", dict(d=0), UNSUPPORTED), ("vp_embed", dict(d=4097, stride=4097), UNSUPPORTED), ("vp_embed", dict(V=0), UNSUPPORTED),
    ("vp_embed", dict(n=-1), UNSUPPORTED), ("vp_embed", dict(n=1 << 31), UNSUPPORTED), ("vp_embed", dict(n=0, table=None), OK),
    ("vp_embed_grad", dict(dout=None), INVALID), ("vp_embed_grad", dict(grad=None), INVALID), ("vp_embed_grad", dict(ws=None), INVALID),
    ("vp_embed_grad", dict(ws=A + 128), INVALID), ("vp_embed_grad", dict(ws_bytes=1000), WORKSPACE), ("vp_embed_grad", dict(dout_type=7), INVALID),
    ("vp_embed_grad", dict(stride=10), INVALID), ("vp_embed_grad", dict(n=-5), UNSUPPORTED), ("vp_embed_grad", dict(grad=A + 2), INVALID),
    ("vp_add_norm", dict(x=None), INVALID), ("vp_add_norm", dict(weight=None), INVALID), ("vp_add_norm", dict(type=5), INVALID),
    ("vp_add_norm", dict(norm_type=9), INVALID), ("vp_add_norm", dict(q=None), INVALID), ("vp_add_norm", dict(scales=None), INVALID),
    ("vp_add_norm", dict(q=A + 4), INVALID), ("vp_add_norm", dict(eps=-1.0), INVALID), ("vp_add_norm", dict(eps=float("nan")), INVALID),
    ("vp_add_norm", dict(x_stride=63), INVALID), ("vp_add_norm", dict(r_stride=63), INVALID), ("vp_add_norm", dict(d=5000, x_stride=5000, r_stride=5000), UNSUPPORTED),
    ("vp_add_norm", dict(n=0, x=None), OK), ("vp_add_norm", dict(n=-1), UNSUPPORTED),
    ("vp_add_norm_grad", dict(dnorm=None), INVALID), ("vp_add_norm_grad", dict(dweight=None), INVALID), ("vp_add_norm_grad", dict(rstd=None), INVALID),
    ("vp_add_norm_grad", dict(ws_bytes=16), WORKSPACE), ("vp_add_norm_grad", dict(ws=A + 64), INVALID), ("vp_add_norm_grad", dict(type=3), INVALID),
    ("vp_add_norm_grad", dict(ds_stride=3), INVALID), ("vp_add_norm_grad", dict(d=0), UNSUPPORTED),
    ("vp_scaled_pack", dict(wq=None), INVALID), ("vp_scaled_pack", dict(packed=A + 16), INVALID), ("vp_scaled_pack", dict(packed_bytes=100), WORKSPACE),
    ("vp_scaled_pack", dict(M=0), UNSUPPORTED), ("vp_scaled_pack", dict(d=16385, stride=16385), UNSUPPORTED), ("vp_scaled_pack", dict(stride=1), INVALID),
    ("vp_scaled_matmul", dict(packed=None), INVALID), ("vp_scaled_matmul", dict(xq=None), INVALID), ("vp_scaled_matmul", dict(out_type=3), INVALID),
    ("vp_scaled_matmul", dict(bias_type=4), INVALID), ("vp_scaled_matmul", dict(bias=A + 1), INVALID), ("vp_scaled_matmul", dict(stride=8), INVALID),
    ("vp_scaled_matmul", dict(ws_bytes=8), WORKSPACE), ("vp_scaled_matmul", dict(ws=A + 8), INVALID), ("vp_scaled_matmul", dict(n=65537), UNSUPPORTED),
    ("vp_scaled_matmul", dict(n=0, xq=None), OK),
    ("vp_beam_select", dict(logits=None), INVALID), ("vp_beam_select", dict(scores=None), INVALID), ("vp_beam_select", dict(out_token=None), INVALID),
    ("vp_beam_select", dict(type=3), INVALID), ("vp_beam_select", dict(stride=99), INVALID), ("vp_beam_select", dict(a_stride=3), INVALID),
    ("vp_beam_select", dict(B=33), UNSUPPORTED), ("vp_beam_select", dict(B=0), UNSUPPORTED), ("vp_beam_select", dict(V=0), UNSUPPORTED),
    ("vp_beam_select", dict(S=65536), UNSUPPORTED), ("vp_beam_select", dict(ws_bytes=8), WORKSPACE), ("vp_beam_select", dict(ws=A + 1), INVALID),
    ("vp_beam_select", dict(logits=A + 1), INVALID), ("vp_beam_select", dict(S=0, logits=None), OK),
])
def test_calls_are_refused_on_the_host(name, kw, status):
    assert _call(name, **kw) == status, vp.last_error()
    assert status == OK or vp.last_error()


def _state(sizes, strides, row_dim=0, elem=2, data=A):
    k = len(sizes)
    pad = lambda v: (ctypes.c_int64 * 8)(*v)  # noqa: E731
    return layers.State(data, elem, k, row_dim, pad(sizes), pad(strides))


@pytest.mark.parametrize("state,kw,status,text", [
    (_state([6, 8], [8, 1]), dict(B=33, S=1), UNSUPPORTED, "B = 33"),
    (_state([6, 8], [8, 1], elem=3), {}, INVALID, "elements"),
    (_state([6, 8], [8, 1], row_dim=2), {}, INVALID, "dimensions"),
    (_state([5, 8], [8, 1]), {}, INVALID, "rows"),
    (_state([6, 8], [8, 0]), {}, INVALID, "overlaps"),
    (_state([6, 8], [4, 1]), {}, INVALID, "overlaps"),
    (_state([6, 8], [-8, 1]), {}, INVALID, "negative"),
    (_state([6, 8], [8, 1], data=None), {}, INVALID, "address"),
    (_state([6, 8], [8, 1], data=A + 1), {}, INVALID, "address"),
    (_state([6, 2, 2, 2, 2, 2], [1000, 2, 8, 32, 128, 512]), {}, UNSUPPORTED, "dimensions"),
    (_state([6, 1 << 20, 1 << 14], [1 << 36, 1 << 16, 2]), {}, UNSUPPORTED, "large"),
    (_state([6, 0], [8, 1], data=None), {}, OK, ""),
    (_state([6, 8], [8, 1]), dict(parent=None), INVALID, "null"),
    (_state([6, 8], [8, 1]), dict(count=9), UNSUPPORTED, "at most"),
    (_state([6, 8], [8, 1]), dict(S=6, B=1), OK, ""),
])
def test_reorder_is_refused_on_the_host(state, kw, status, text):
    a = dict(dict(count=1, parent=A, S=2, B=3), **kw)
    assert vp.lib().vp_beam_reorder(ctypes.byref(state), a["count"], a["parent"], a["S"], a["B"], None) == status, vp.last_error()
    assert text in vp.last_error() or status == OK


def test_workspace_sizes():
    L = vp.lib()
    assert L.vp_embed_grad_workspace_bytes(1000, 100, 64) > 0 and L.vp_embed_grad_workspace_bytes(0, 100, 64) > 0
    assert L.vp_embed_grad_workspace_bytes(-1, 100, 64) == 0 and L.vp_embed_grad_workspace_bytes(10, 100, 5000) == 0
    assert L.vp_embed_grad_workspace_bytes(2000, 100, 64) >= L.vp_embed_grad_workspace_bytes(1000, 100, 64)
    assert L.vp_add_norm_grad_workspace_bytes(10, 64) > 0 and L.vp_add_norm_grad_workspace_bytes(10, 0) == 0
    assert L.vp_scaled_pack_bytes(100, 64) >= 128 * 128 and L.vp_scaled_pack_bytes(0, 64) == 0
    assert L.vp_scaled_matmul_workspace_bytes(5, 64) > 0 and L.vp_scaled_matmul_workspace_bytes(5, 1 << 20) == 0
    assert L.vp_beam_select_workspace_bytes(2, 3, 100) > 0 and L.vp_beam_select_workspace_bytes(2, 40, 100) == 0


def test_binding_refuses_host_tensors_and_wrong_types_before_any_c_call():
    h, f = torch.zeros((6, 64), dtype=torch.float16), torch.zeros(6)
    ids = torch.zeros(6, dtype=torch.int32)
    for call in (lambda: P.vp_embed(h, ids), lambda: P.vp_embed_grad(h, ids, 10), lambda: P.vp_add_norm(h, h[0]),
                 lambda: P.vp_add_norm_grad(h, h, h[0], f), lambda: P.vp_scaled_pack(h.to(torch.float8_e4m3fn), torch.ones(1, 1)),
                 lambda: P.vp_beam_select(h, f, 3), lambda: P.vp_beam_reorder([(h, 0)], ids, 3)):
        with pytest.raises(ValueError, match="GPU memory"):
            call()
    with pytest.raises(TypeError):
        P.vp_scaled_matmul(h, h, f)
    with pytest.raises(TypeError):
        P.vp_embed([1, 2], ids)
    with pytest.raises(ValueError, match="two dimensions"):
        P.vp_embed(f, ids)
    with pytest.raises(ValueError, match="float8"):
        P.vp_scaled_pack(h, torch.ones(1, 1))
    with pytest.raises(ValueError, match="one of"):
        layers._type_code(torch.float64, "t")


@pytest.mark.parametrize("state,kw,status", [
    (_state([6, 8], [8, 1]), {}, OK), (_state([6, 8], [8, 0]), {}, INVALID), (_state([5, 8], [8, 1]), {}, INVALID), (_state([6, 8], [8, 1], elem=3), {}, INVALID),
    (_state([6, 2, 2, 2, 2, 2], [1000, 2, 8, 32, 128, 512]), {}, UNSUPPORTED), (_state([6, 8], [8, 1]), dict(count=9), UNSUPPORTED),
    (_state([6, 8], [8, 1]), dict(B=33, S=1), UNSUPPORTED), (_state([6, 8], [8, 1], data=None), dict(count=0), OK)])
def test_reorder_check_says_what_reorder_would(state, kw, status):
    a = dict(dict(count=1, S=2, B=3), **kw)
    assert vp.lib().vp_beam_reorder_check(ctypes.byref(state), a["count"], a["S"], a["B"]) == status, vp.last_error()
    if status != OK:
        said = vp.last_error()
        assert vp.lib().vp_beam_reorder(ctypes.byref(state), a["count"], A, a["S"], a["B"], None) == status and vp.last_error() == said
    assert vp.lib().vp_beam_reorder_check(None, 1, 2, 3) == INVALID


def test_selection_refuses_more_pieces_than_a_launch_has_threads():
    """A row is cut into pieces of 8,192 fp32 or 12,288 16-bit values, a workgroup of 256 threads each; a launch has less than 2^32."""
    most = 1 << 24
    for code, width in ((0, 12288), (1, 12288), (2, 8192)):
        for S, V in ((32768, width * (most // 65536) + 1), (8192, 1 << 30)):
            kw = dict(type=code, S=S, B=2, V=V, stride=V, a_stride=-(-V // 32), ws_bytes=1 << 50)
            assert _call("vp_beam_select", **kw) == UNSUPPORTED and "too many" in vp.last_error()


@pytest.mark.parametrize("kw", [dict(x_stride=65), dict(r_stride=65), dict(x_stride=1000, residual=A + 0x100000), dict(r_stride=64 + 8, x=A + 0x100000)])
def test_norm_refuses_a_sum_over_rows_that_are_apart(kw):
    assert _call("vp_add_norm", **kw) == INVALID and "contiguous" in vp.last_error()


@pytest.mark.parametrize("state", [_state([2, 1 << 61], [1 << 61, 1], elem=8), _state([2, 1 << 62], [1 << 62, 1], elem=4), _state([2, 3, 1 << 40], [1, 1 << 62, 2]),
                                   _state([2, 1 << 49], [1, 2], elem=1)])
def test_reorder_refuses_sizes_past_any_memory(state):
    """Their products leave 64 bits: nothing may be made of what is left of them."""
    assert vp.lib().vp_beam_reorder_check(ctypes.byref(state), 1, 1, 2) == INVALID and "memory" in vp.last_error()
