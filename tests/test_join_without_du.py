"""Without the gradient at u the join's backward call goes as far as o: the norm before u, x and o
are not looked at."""
import pytest
import torch

import paper_1903_06681_amd as dc
import test_gpu_act as T
import test_gpu_block_ops as B
from test_act_host import MIS16, Ws, view
from test_block_host import P1, P2, P3, P4, with_

V = dc.View.of
BAD = [dc.Norm(9, 1e-5), dc.Norm(dc.DC_NORM_LAYER, float("nan")), dc.Norm(dc.DC_NORM_RMS, 1e-5, MIS16), dc.Norm(dc.DC_NORM_RMS, 1e-5, None, MIS16)]


@pytest.mark.parametrize("k", range(len(BAD)))
def test_no_refusal_for_what_is_not_looked_at(k):
    """A call that goes on to what it does look at: it is refused for its workspace."""
    v, w = view(), view(C=9)
    call = with_(dc.join_bwd, dict(vdu=None, du=None, vdo=v, do=P1, vy=v, y=P2, vx=w, x=MIS16, vo=w, o=MIS16, stat=P4, post=None, scale=None,
                                   gate=None, drop=None, pre=BAD[k], vdx=v, dx=P3, vdy=v, dy=P4, grads=dc.JoinGrads(scale=P1), accumulate=0,
                                   workspace=Ws(0), stream=0))
    assert call() == -6
    assert call(vdu=v, du=P1, vx=v, vo=None, o=None) in (-10, -7)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,layout", [((2, 40, 9, 11), "dense"), ((5, 130, 7, 1), "rows"), ((2, 2100, 3, 4), "gaps")], ids=str)
def test_results_do_not_depend_on_it(shape, layout):
    N, C, H, W = shape
    g = T.rng(22)
    y, do = (T.put(layout, T.randn(g, *shape), "f32")[0] for _ in range(2))
    post, stat = dc.Norm(dc.DC_NORM_LAYER, B.EPS), T.randn(g, 4, N, H, W).abs().cuda()
    par = B.vec(g, C + 1)
    found = []
    for pre, x in ((None, None), (dc.Norm(9, float("nan"), par[1:], par[1:]), do)):
        grads = dc.JoinGrads(scale=torch.empty(C, device="cuda"), gamma_post=torch.empty(C, device="cuda"))
        dx, dy, mem = torch.empty_like(do), torch.empty_like(y), T.ws(dc.join_bwd_workspace_bytes(V(y), False))
        vx = V(x) if x is not None else None
        dc.join_bwd(None, None, V(do), do, V(y), y, vx, x, vx, x, stat, post, None, None, None, pre, V(dx), dx, V(dy), dy, grads, 0, mem)
        found.append([dx, dy, grads.scale, grads.gamma_post])
    for a, b in zip(*found):
        assert torch.equal(a, b)
    assert torch.equal(found[0][0], do)
