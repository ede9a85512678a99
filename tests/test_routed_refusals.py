"""What the routed layer's operators refuse: by the C ABI on the host, before any HIP call, and by
the Python functions. No GPU needed."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2308_11825_amd as agcn

F, B, H = agcn.AGCN_FLOAT, agcn.AGCN_BFLOAT, agcn.AGCN_HALF
BAD, UNSUPPORTED = agcn.AGCN_ERR_INVALID_ARGUMENT, agcn.AGCN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return agcn.load_library()


def _with(base, **change):
    args = dict(base, **change)
    assert set(args) == set(base)
    return list(args.values())


NORM = dict(n=8, f=200, dtype=B, X=0x100000, ldx=200, R=0x110000, ldr=200, Hid=0x120000, ldh=200, g=0x130000,
            b=0x140000, p_dtype=F, eps=1e-6, Y=0x200000, ldy=200, stats=0x300000, lds=2, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(f=-1), BAD), (dict(dtype=4), BAD), (dict(p_dtype=H), BAD), (dict(dtype=F, p_dtype=B), BAD),
    (dict(eps=0.0), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("inf")), BAD), (dict(eps=float("nan")), BAD),
    (dict(X=None), BAD), (dict(g=None), BAD), (dict(Y=None), BAD), (dict(ldx=199), BAD), (dict(ldr=199), BAD),
    (dict(ldh=199), BAD), (dict(ldy=199), BAD), (dict(lds=1), BAD), (dict(Hid=0x100000, ldh=204), BAD),
    (dict(Hid=0x110190), BAD), (dict(Y=0x100000), BAD), (dict(Y=0x110000), BAD), (dict(Y=0x120000), BAD),
    (dict(Y=0x130000), BAD), (dict(Y=0x140000), BAD), (dict(stats=0x200000), BAD), (dict(stats=0x100000), BAD),
    (dict(X=0x100001), BAD), (dict(g=0x130002), BAD), (dict(b=0x140002), BAD), (dict(stats=0x300002), BAD),
    (dict(ldx=2 ** 61), BAD),
    (dict(f=2 ** 24 + 1, ldx=2 ** 25, ldr=2 ** 25, ldh=2 ** 25, ldy=2 ** 25), UNSUPPORTED),
    (dict(n=0, X=None, R=None, Hid=None, Y=None, stats=None), 0),
    (dict(f=0, X=None, R=None, Hid=None, g=None, b=None, Y=None, stats=None), 0)])
def test_layer_norm(lib, change, status):
    assert lib.agcn_layer_norm(*_with(NORM, **change)) == status, agcn.agcn_last_error()


GRAD = dict(n=8, f=200, dtype=B, dY=0x100000, lddy=200, Hid=0x110000, ldh=200, dH=0x120000, lddh=200, stats=0x130000,
            lds=2, g=0x140000, p_dtype=F, dX=0x200000, lddx=200, dg=0x210000, db=0x220000, ws=0x300000, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(f=-1), BAD), (dict(dtype=3), BAD), (dict(p_dtype=H), BAD), (dict(dY=None), BAD),
    (dict(Hid=None), BAD), (dict(stats=None), BAD), (dict(g=None), BAD), (dict(dX=None), BAD), (dict(ws=None), BAD),
    (dict(lddy=199), BAD), (dict(ldh=199), BAD), (dict(lddh=199), BAD), (dict(lddx=199), BAD), (dict(lds=1), BAD),
    (dict(dX=0x100000), BAD), (dict(dX=0x110000), BAD), (dict(dX=0x120000), BAD), (dict(dX=0x130000), BAD),
    (dict(dX=0x140000), BAD), (dict(dg=0x140000), BAD), (dict(db=0x210000), BAD), (dict(ws=0x200000), BAD),
    (dict(ws=0x130000), BAD), (dict(ws=0x300002), BAD), (dict(dg=0x210002), BAD), (dict(dX=0x200001), BAD),
    (dict(f=2 ** 24 + 1, lddy=2 ** 25, ldh=2 ** 25, lddh=2 ** 25, lddx=2 ** 25), UNSUPPORTED),
    (dict(f=0, dY=None, Hid=None, dH=None, stats=None, g=None, dX=None, dg=None, db=None, ws=None), 0),
    (dict(n=0, dY=None, Hid=None, dH=None, stats=None, g=None, dX=None, dg=None, db=None, ws=None), 0)])
def test_layer_norm_backward(lib, change, status):
    assert lib.agcn_layer_norm_backward(*_with(GRAD, **change)) == status, agcn.agcn_last_error()


SORT = dict(n=100000, k=4, groups=64, ids=0x1000000, id_bytes=4, ldi=4, offsets=0x2000000, place=0x3000000, ldp=4,
            ws=0x4000000, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(k=-1), BAD), (dict(groups=-1), BAD), (dict(id_bytes=2), BAD), (dict(id_bytes=0), BAD),
    (dict(ids=None), BAD), (dict(offsets=None), BAD), (dict(place=None), BAD), (dict(ws=None), BAD), (dict(ldi=3), BAD),
    (dict(ldp=3), BAD), (dict(ids=0x1000002), BAD), (dict(id_bytes=8, ids=0x1000004), BAD), (dict(place=0x1000000), BAD),
    (dict(offsets=0x3000000), BAD), (dict(ws=0x2000000), BAD), (dict(ws=0x4000002), BAD),
    (dict(groups=65537), UNSUPPORTED), (dict(n=2 ** 31), UNSUPPORTED), (dict(n=2 ** 29), UNSUPPORTED),
    (dict(n=2 ** 30, k=3), UNSUPPORTED)])
def test_sort_groups(lib, change, status):
    assert lib.agcn_sort_groups(*_with(SORT, **change)) == status, agcn.agcn_last_error()


def test_workspace_sizes(lib):
    assert agcn.agcn_sort_groups_workspace_size(8, 4, 64) == 0
    assert agcn.agcn_sort_groups_workspace_size(0, 0, 1000) == 0
    big = agcn.agcn_sort_groups_workspace_size(2 ** 31 - 1, 1, 65536)
    assert 0 < big <= 257 * 65537 * 4
    assert agcn.agcn_layer_norm_workspace_size(0, 100, F) == 0 and agcn.agcn_layer_norm_workspace_size(5, 0, F) == 0
    for n, f in ((1, 1), (1000, 128), (2 ** 40, 4096), (100, 2 ** 24)):
        for t in (F, B, H):
            assert agcn.agcn_layer_norm_workspace_size(n, f, t) % (8 * f) == 0
    b = ctypes.c_size_t()
    for call in (lambda: lib.agcn_sort_groups_workspace_size(-1, 1, 1, ctypes.byref(b)),
                 lambda: lib.agcn_sort_groups_workspace_size(1, 1, -1, ctypes.byref(b)),
                 lambda: lib.agcn_sort_groups_workspace_size(1, 1, 1, None),
                 lambda: lib.agcn_layer_norm_workspace_size(-1, 1, F, ctypes.byref(b)),
                 lambda: lib.agcn_layer_norm_workspace_size(1, -1, F, ctypes.byref(b)),
                 lambda: lib.agcn_layer_norm_workspace_size(1, 1, 9, ctypes.byref(b)),
                 lambda: lib.agcn_layer_norm_workspace_size(1, 1, F, None)):
        assert call() == BAD
    assert lib.agcn_sort_groups_workspace_size(1, 1, 65537, ctypes.byref(b)) == UNSUPPORTED
    assert lib.agcn_layer_norm_workspace_size(1, 2 ** 24 + 1, F, ctypes.byref(b)) == UNSUPPORTED


DISPATCH = dict(n=8, k=2, bytes=400, X=0x100000, ldx=400, place=0x110000, ldp=2, Y=0x200000, ldy=400, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(k=-1), BAD), (dict(bytes=-1), BAD), (dict(X=None), BAD), (dict(place=None), BAD),
    (dict(Y=None), BAD), (dict(ldx=399), BAD), (dict(ldp=1), BAD), (dict(ldy=399), BAD), (dict(place=0x110002), BAD),
    (dict(Y=0x100000), BAD), (dict(Y=0x110000), BAD), (dict(bytes=2 ** 27 + 1, ldx=2 ** 28, ldy=2 ** 28), UNSUPPORTED),
    (dict(n=2 ** 30, k=2), UNSUPPORTED), (dict(n=0, X=None, place=None, Y=None), 0),
    (dict(k=0, X=None, place=None, Y=None), 0), (dict(bytes=0, X=None, place=None, Y=None), 0)])
def test_dispatch(lib, change, status):
    assert lib.agcn_dispatch(*_with(DISPATCH, **change)) == status, agcn.agcn_last_error()


COMBINE = dict(n=8, k=2, f=200, dtype=B, R=0x100000, ldr=200, place=0x110000, ldp=2, W=0x120000, ldw=2, Y=0x200000,
               ldy=200, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(k=-1), BAD), (dict(f=-1), BAD), (dict(dtype=3), BAD), (dict(R=None), BAD),
    (dict(place=None), BAD), (dict(Y=None), BAD), (dict(ldr=199), BAD), (dict(ldp=1), BAD), (dict(ldw=1), BAD),
    (dict(ldy=199), BAD), (dict(Y=0x100000), BAD), (dict(Y=0x110000), BAD), (dict(Y=0x120000), BAD),
    (dict(W=0x120002), BAD), (dict(R=0x100001), BAD), (dict(f=2 ** 24 + 1, ldr=2 ** 25, ldy=2 ** 25), UNSUPPORTED),
    (dict(n=2 ** 30, k=2), UNSUPPORTED), (dict(n=0, R=None, place=None, W=None, Y=None), 0),
    (dict(f=0, R=None, place=None, W=None, Y=None), 0)])
def test_combine(lib, change, status):
    assert lib.agcn_combine(*_with(COMBINE, **change)) == status, agcn.agcn_last_error()


COMBINE_GRAD = dict(n=8, k=2, f=200, dtype=B, dY=0x100000, lddy=200, R=0x110000, ldr=200, place=0x120000, ldp=2,
                    W=0x130000, ldw=2, dR=0x200000, lddr=200, dW=0x210000, lddw=2, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(k=-1), BAD), (dict(f=-1), BAD), (dict(dtype=3), BAD), (dict(dY=None), BAD),
    (dict(R=None), BAD), (dict(place=None), BAD), (dict(W=None), BAD), (dict(dR=None), BAD), (dict(dW=None), BAD),
    (dict(lddy=199), BAD), (dict(ldr=199), BAD), (dict(ldp=1), BAD), (dict(ldw=1), BAD), (dict(lddr=199), BAD),
    (dict(lddw=1), BAD), (dict(dR=0x100000), BAD), (dict(dR=0x110000), BAD), (dict(dW=0x130000), BAD),
    (dict(dW=0x200000), BAD), (dict(dW=0x210002), BAD), (dict(n=2 ** 30, k=2), UNSUPPORTED),
    (dict(n=0, dY=None, R=None, place=None, W=None, dR=None, dW=None), 0),
    (dict(k=0, dY=None, R=None, place=None, W=None, dR=None, dW=None), 0)])
def test_combine_backward(lib, change, status):
    assert lib.agcn_combine_backward(*_with(COMBINE_GRAD, **change)) == status, agcn.agcn_last_error()


ROWS = dict(n=8, f=200, dtype=F, X=0x100000, ldx=200, Q=0x200000, ldq=208, S=0x300000, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(f=-1), BAD), (dict(dtype=3), BAD), (dict(X=None), BAD), (dict(Q=None), BAD),
    (dict(S=None), BAD), (dict(ldx=199), BAD), (dict(ldq=199), BAD), (dict(X=0x100002), BAD), (dict(S=0x300002), BAD),
    (dict(Q=0x100010), BAD), (dict(S=0x200100), BAD), (dict(f=2 ** 24 + 1, ldx=2 ** 25, ldq=2 ** 25), UNSUPPORTED),
    (dict(n=0, X=None, Q=None, S=None), 0)])
def test_quantize_rows_int(lib, change, status):
    assert lib.agcn_quantize_rows_int(*_with(ROWS, **change)) == status, agcn.agcn_last_error()


WEIGHT = dict(groups=2, fin=200, fout=130, dtype=B, W=0x1000000, ldw=130, group_w=26000, Q=0x2000000, ldq=208,
              group_q=27040, S=0x3000000, group_s=130, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(groups=-1), BAD), (dict(fin=-1), BAD), (dict(fout=-1), BAD), (dict(dtype=7), BAD), (dict(ldw=129), BAD),
    (dict(ldq=199), BAD), (dict(group_w=-1), BAD), (dict(group_q=27000), BAD), (dict(group_s=129), BAD),
    (dict(W=None), BAD), (dict(Q=None), BAD), (dict(S=None), BAD), (dict(Q=0x1000000), BAD), (dict(S=0x2000010), BAD),
    (dict(W=0x1000001), BAD), (dict(S=0x3000001), BAD), (dict(groups=2 ** 24 + 1), UNSUPPORTED),
    (dict(groups=0, W=None, Q=None, S=None), 0), (dict(fout=0, ldw=0, W=None, Q=None, S=None), 0)])
def test_quantize_weight_int(lib, change, status):
    assert lib.agcn_quantize_weight_int(*_with(WEIGHT, **change)) == status, agcn.agcn_last_error()


LINEAR = dict(n=8, fin=200, fout=130, Q=0x100000, ldq=208, S=0x110000, WQ=0x200000, ldwq=208, WS=0x300000, dtype=B,
              Y=0x400000, ldy=130, stream=None, epilogue=0)
GROUPED = dict(n=8, fin=200, fout=130, groups=3, Q=0x100000, ldq=208, S=0x110000, WQ=0x200000, ldwq=208, group_wq=27040,
               WS=0x300000, group_ws=130, offsets=0x310000, dtype=B, Y=0x400000, ldy=130, stream=None, epilogue=0)
BOTH = [
    (dict(n=-1), BAD), (dict(fin=-1), BAD), (dict(fout=-1), BAD), (dict(dtype=5), BAD), (dict(epilogue=2), BAD),
    (dict(ldq=199), BAD), (dict(ldwq=199), BAD), (dict(ldy=129), BAD), (dict(Q=None), BAD), (dict(S=None), BAD),
    (dict(WQ=None), BAD), (dict(WS=None), BAD), (dict(Y=None), BAD), (dict(Y=0x400001), BAD), (dict(S=0x110002), BAD),
    (dict(WS=0x300002), BAD), (dict(Y=0x100100), BAD), (dict(Y=0x200100), BAD), (dict(Y=0x300000), BAD),
    (dict(Y=0x110000), BAD), (dict(fin=2 ** 17, ldq=2 ** 17, ldwq=2 ** 17), UNSUPPORTED),
    (dict(fout=2 ** 24 + 1, ldy=2 ** 25), UNSUPPORTED), (dict(n=0, Q=None, S=None, WQ=None, WS=None, Y=None), 0),
    (dict(fout=0, ldy=0, Q=None, S=None, WQ=None, WS=None, Y=None), 0)]


@pytest.mark.parametrize("change,status", BOTH)
def test_int_linear(lib, change, status):
    assert lib.agcn_int_linear(*_with(LINEAR, **change)) == status, agcn.agcn_last_error()


@pytest.mark.parametrize("change,status", BOTH + [
    (dict(groups=-1), BAD), (dict(offsets=None), BAD), (dict(offsets=0x310002), BAD), (dict(Y=0x310000), BAD),
    (dict(group_wq=-16), BAD), (dict(group_ws=-1), BAD), (dict(n=2 ** 31), UNSUPPORTED),
    (dict(groups=2 ** 24 + 1), UNSUPPORTED)])
def test_grouped_int_linear(lib, change, status):
    assert lib.agcn_grouped_int_linear(*_with(GROUPED, **change)) == status, agcn.agcn_last_error()


def test_python_refuses_what_is_not_on_a_gpu():
    x, g, s = torch.zeros(4, 8), torch.ones(8), torch.zeros(4, 2)
    q, i = torch.zeros((4, 8), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.int32)
    off = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: agcn.layer_norm(x, g), lambda: agcn.layer_norm(None, g),
                 lambda: agcn.layer_norm_backward(x, x, s, g), lambda: agcn.layer_norm_backward(None, x, s, g),
                 lambda: agcn.sort_groups(i, 3), lambda: agcn.sort_groups(None, 3), lambda: agcn.dispatch(x, i),
                 lambda: agcn.dispatch(None, i), lambda: agcn.combine(x, i), lambda: agcn.combine(x, None),
                 lambda: agcn.combine_backward(x, x, i, s), lambda: agcn.quantize_int(x),
                 lambda: agcn.quantize_int(None), lambda: agcn.quantize_weight_int(x),
                 lambda: agcn.int_linear(q, s, q, s), lambda: agcn.grouped_int_linear(q, s, q[None], s[None], off),
                 lambda: agcn.grouped_int_linear(q, s, q[None], s[None], [0, 4])):
        with pytest.raises((TypeError, ValueError)):
            call()
