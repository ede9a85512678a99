"""The functions with the C names of the routed layer's operators: the Python functions' results,
with plain addresses, strides and workspaces."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import randn  # noqa: E402

DEV = "cuda:0"
F, B = agcn.AGCN_FLOAT, agcn.AGCN_BFLOAT


def workspace(nbytes):
    ws = torch.empty(max(nbytes, 4) // 4, dtype=torch.int32, device=DEV)
    return ws, ws.data_ptr() if nbytes else None


def test_layer_norm():
    n, f = 40, 200
    x, r, dy, dh = (randn((n, f), torch.bfloat16, i) for i in range(4))
    g, b = randn((f,), torch.float32, 5), randn((f,), torch.float32, 6)
    y, h, stats = agcn.layer_norm(x, g, b, residual=r, stats=True)
    Y, H, S = torch.empty_like(y), torch.empty_like(h), torch.empty_like(stats)
    st = torch.cuda.current_stream().cuda_stream
    agcn.agcn_layer_norm(n, f, B, x.data_ptr(), f, r.data_ptr(), f, H.data_ptr(), f, g.data_ptr(), b.data_ptr(), F, 1e-5,
                         Y.data_ptr(), f, S.data_ptr(), 2, st)
    assert torch.equal(Y, y) and torch.equal(H, h) and torch.equal(S, stats)
    want = agcn.layer_norm_backward(dy, h, stats, g, grad_hidden=dh)
    got = [torch.empty_like(t) for t in want]
    ws, at = workspace(agcn.agcn_layer_norm_workspace_size(n, f, B))
    agcn.agcn_layer_norm_backward(n, f, B, dy.data_ptr(), f, H.data_ptr(), f, dh.data_ptr(), f, S.data_ptr(), 2,
                                  g.data_ptr(), F, got[0].data_ptr(), f, got[1].data_ptr(), got[2].data_ptr(), at, st)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    # Neither sum, without a workspace; and one of them alone.
    only = torch.empty_like(want[0])
    agcn.agcn_layer_norm_backward(n, f, B, dy.data_ptr(), f, H.data_ptr(), f, dh.data_ptr(), f, S.data_ptr(), 2,
                                  g.data_ptr(), F, only.data_ptr(), f, None, None, None, st)
    assert torch.equal(only, want[0])
    db = torch.empty_like(want[2])
    agcn.agcn_layer_norm_backward(n, f, B, dy.data_ptr(), f, H.data_ptr(), f, None, 0 + f, S.data_ptr(), 2, g.data_ptr(), F,
                                  only.data_ptr(), f, None, db.data_ptr(), at, st)
    assert torch.equal(db, want[2])


@pytest.mark.parametrize("n,k,groups,ids_dtype", [(30, 3, 7, torch.int32), (20000, 2, 40, torch.int64)])
def test_rows_there_and_back(n, k, groups, ids_dtype):
    f = 24
    ids = (torch.arange(n * k, device=DEV) * 7919 % (groups + 1)).view(n, k).to(ids_dtype)
    offsets, place = agcn.sort_groups(ids, groups)
    O, P = torch.empty_like(offsets), torch.empty_like(place)
    st = torch.cuda.current_stream().cuda_stream
    ws, at = workspace(agcn.agcn_sort_groups_workspace_size(n, k, groups))
    agcn.agcn_sort_groups(n, k, groups, ids.data_ptr(), ids.element_size(), k, O.data_ptr(), P.data_ptr(), k, at, st)
    assert torch.equal(O, offsets) and torch.equal(P, place)
    x, w, dy = randn((n, f), torch.bfloat16, 1), randn((n, k), torch.float32, 2), randn((n, f), torch.bfloat16, 3)
    rows = agcn.dispatch(x, place)
    R = torch.empty_like(rows)
    agcn.agcn_dispatch(n, k, 2 * f, x.data_ptr(), 2 * f, P.data_ptr(), k, R.data_ptr(), 2 * f, st)
    assert torch.equal(R, rows)
    out = agcn.combine(rows, place, w)
    Y = torch.empty_like(out)
    agcn.agcn_combine(n, k, f, B, R.data_ptr(), f, P.data_ptr(), k, w.data_ptr(), k, Y.data_ptr(), f, st)
    assert torch.equal(Y, out)
    agcn.agcn_combine(n, k, f, B, R.data_ptr(), f, P.data_ptr(), k, None, k, Y.data_ptr(), f, st)
    assert torch.equal(Y, agcn.combine(rows, place))
    dR, dw = agcn.combine_backward(dy, rows, place, w)
    got = torch.empty_like(dR), torch.empty_like(dw)
    agcn.agcn_combine_backward(n, k, f, B, dy.data_ptr(), f, R.data_ptr(), f, P.data_ptr(), k, w.data_ptr(), k,
                               got[0].data_ptr(), f, got[1].data_ptr(), k, st)
    assert torch.equal(got[0], dR) and torch.equal(got[1], dw)


def test_integers():
    n, fin, fout, e = 50, 96, 20, 2
    x, W = randn((n, fin), torch.bfloat16, 1), randn((e, fin, fout), torch.bfloat16, 2)
    q, s = agcn.quantize_int(x)
    wq, ws = agcn.quantize_weight_int(W)
    st = torch.cuda.current_stream().cuda_stream
    Q, S = torch.empty((n, fin), dtype=torch.int8, device=DEV), torch.empty_like(s)
    agcn.agcn_quantize_rows_int(n, fin, B, x.data_ptr(), fin, Q.data_ptr(), fin, S.data_ptr(), st)
    assert torch.equal(Q, q) and torch.equal(S, s)
    WQ, WS = torch.empty((e, fout, fin), dtype=torch.int8, device=DEV), torch.empty_like(ws)
    agcn.agcn_quantize_weight_int(e, fin, fout, B, W.data_ptr(), fout, fin * fout, WQ.data_ptr(), fin, fin * fout,
                                  WS.data_ptr(), fout, st)
    assert torch.equal(WQ, wq) and torch.equal(WS, ws)
    Y = torch.empty((n, fout), dtype=torch.bfloat16, device=DEV)
    agcn.agcn_int_linear(n, fin, fout, Q.data_ptr(), fin, S.data_ptr(), WQ.data_ptr(), fin, WS.data_ptr(), B, Y.data_ptr(),
                         fout, st, agcn.AGCN_EPILOGUE_RELU)
    assert torch.equal(Y, agcn.int_linear(q, s, wq[0], ws[0], dtype=torch.bfloat16, act="relu"))
    offsets = torch.tensor([3, 20, 45], dtype=torch.int32, device=DEV)
    agcn.agcn_grouped_int_linear(n, fin, fout, e, Q.data_ptr(), fin, S.data_ptr(), WQ.data_ptr(), fin, fin * fout,
                                 WS.data_ptr(), fout, offsets.data_ptr(), B, Y.data_ptr(), fout, st)
    assert torch.equal(Y, agcn.grouped_int_linear(q, s, wq, ws, offsets, dtype=torch.bfloat16))
