"""What the 8-bit operators refuse: by the C ABI on the host, before any HIP call, and
by the Python functions. No GPU needed."""
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


ROWS = dict(n=8, f=200, dtype=F, X=0x100000, ldx=200, Q=0x200000, ldq=208, S=0x300000, lds=2,
            stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(f=-1), BAD), (dict(f=2 ** 24 + 1, ldx=2 ** 25, ldq=2 ** 25, lds=2 ** 20),
                                           UNSUPPORTED),
    (dict(dtype=3), BAD), (dict(dtype=-1), BAD), (dict(X=None), BAD), (dict(Q=None), BAD),
    (dict(S=None), BAD), (dict(ldx=199), BAD), (dict(ldq=199), BAD), (dict(lds=1), BAD),
    (dict(X=0x100002), BAD), (dict(ldx=2 ** 61), BAD), (dict(Q=0x100010), BAD), (dict(S=0x200100), BAD),
    (dict(n=0, X=None, Q=None, S=None), 0), (dict(f=0, X=None, Q=None, S=None), 0)])
def test_quantize_rows(lib, change, status):
    assert lib.agcn_quantize_rows(*_with(ROWS, **change)) == status, agcn.agcn_last_error()


WEIGHT = dict(groups=2, fin=200, fout=130, dtype=B, W=0x1000000, ldw=130, group_w=26000, Q=0x2000000,
              ldq=208, group_q=27040, S=0x3000000, lds=2, group_s=4, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(groups=-1), BAD), (dict(fin=-1), BAD), (dict(fout=-1), BAD), (dict(dtype=7), BAD),
    (dict(ldw=129), BAD), (dict(ldq=199), BAD), (dict(lds=1), BAD), (dict(group_w=-1), BAD),
    (dict(group_q=27000), BAD), (dict(group_s=3), BAD), (dict(W=None), BAD), (dict(Q=None), BAD),
    (dict(S=None), BAD), (dict(Q=0x1000000), BAD), (dict(S=0x2000010), BAD), (dict(W=0x1000001), BAD),
    (dict(group_w=2 ** 61), BAD), (dict(groups=0, W=None, Q=None, S=None), 0),
    (dict(fin=0, ldq=0, W=None, Q=None, S=None), 0)])
def test_quantize_weight(lib, change, status):
    assert lib.agcn_quantize_weight(*_with(WEIGHT, **change)) == status, agcn.agcn_last_error()


NORM = dict(n=8, f=200, dtype=B, X=0x100000, ldx=200, R=0x110000, ldr=200, Hid=0x120000, ldh=200,
            g=0x130000, g_dtype=F, eps=1e-6, Q=0x200000, ldq=208, S=0x300000, lds=2, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), BAD), (dict(f=-1), BAD), (dict(dtype=4), BAD), (dict(g_dtype=H), BAD),
    (dict(dtype=F, g_dtype=B), BAD), (dict(eps=0.0), BAD), (dict(eps=-1.0), BAD),
    (dict(eps=float("inf")), BAD), (dict(eps=float("nan")), BAD), (dict(X=None), BAD),
    (dict(g=None), BAD), (dict(Q=None), BAD), (dict(S=None), BAD), (dict(ldx=199), BAD),
    (dict(ldr=199), BAD), (dict(ldh=199), BAD), (dict(ldq=100), BAD), (dict(lds=1), BAD),
    (dict(Hid=0x100000, ldh=204), BAD),          # on X with another stride
    (dict(Hid=0x100002), BAD), (dict(Hid=0x110190), BAD), (dict(Q=0x100000), BAD),
    (dict(Q=0x110000), BAD), (dict(Q=0x120000), BAD), (dict(S=0x200000), BAD), (dict(Q=0x130000), BAD),
    (dict(X=0x100001), BAD), (dict(g=0x130002), BAD),
    (dict(n=0, X=None, R=None, Hid=None, Q=None, S=None), 0)])
def test_rms_norm(lib, change, status):
    assert lib.agcn_rms_norm(*_with(NORM, **change)) == status, agcn.agcn_last_error()


LINEAR = dict(n=8, fin=200, fout=130, Q=0x100000, ldq=208, S=0x110000, lds=2, WQ=0x200000, ldwq=208,
              WS=0x300000, ldws=2, dtype=B, Y=0x400000, ldy=130, stream=None, epilogue=0)
GROUPED = dict(n=8, fin=200, fout=130, groups=3, Q=0x100000, ldq=208, S=0x110000, lds=2, WQ=0x200000,
               ldwq=208, group_wq=27040, WS=0x300000, ldws=2, group_ws=4, offsets=0x310000, dtype=B,
               Y=0x400000, ldy=130, stream=None, epilogue=0)
BOTH = [
    (dict(n=-1), BAD), (dict(fin=-1), BAD), (dict(fout=-1), BAD), (dict(dtype=5), BAD),
    (dict(epilogue=2), BAD), (dict(epilogue=-1), BAD), (dict(ldq=199), BAD), (dict(lds=1), BAD),
    (dict(ldwq=199), BAD), (dict(ldws=1), BAD), (dict(ldy=129), BAD), (dict(Q=None), BAD),
    (dict(S=None), BAD), (dict(WQ=None), BAD), (dict(WS=None), BAD), (dict(Y=None), BAD),
    (dict(Y=0x400001), BAD), (dict(dtype=F, Y=0x400002), BAD), (dict(Y=0x100100), BAD),
    (dict(Y=0x200100), BAD), (dict(Y=0x300000), BAD), (dict(Y=0x110000), BAD), (dict(ldy=2 ** 61), BAD),
    (dict(fin=2 ** 24 + 1, ldq=2 ** 25, lds=2 ** 20, ldwq=2 ** 25, ldws=2 ** 20), UNSUPPORTED),
    (dict(fout=2 ** 24 + 1, ldy=2 ** 25), UNSUPPORTED),
    (dict(n=0, Q=None, S=None, WQ=None, WS=None, Y=None), 0),
    (dict(fout=0, ldy=0, Q=None, S=None, WQ=None, WS=None, Y=None), 0)]


@pytest.mark.parametrize("change,status", BOTH)
def test_quantized_linear(lib, change, status):
    assert lib.agcn_quantized_linear(*_with(LINEAR, **change)) == status, agcn.agcn_last_error()


@pytest.mark.parametrize("change,status", BOTH + [
    (dict(groups=-1), BAD), (dict(offsets=None), BAD), (dict(offsets=0x310002), BAD),
    (dict(Y=0x310000), BAD), (dict(group_wq=-16), BAD), (dict(group_ws=-1), BAD),
    (dict(group_wq=2 ** 61), BAD), (dict(n=2 ** 31), UNSUPPORTED), (dict(groups=2 ** 24 + 1), UNSUPPORTED)])
def test_grouped_linear(lib, change, status):
    assert lib.agcn_grouped_linear(*_with(GROUPED, **change)) == status, agcn.agcn_last_error()


def test_python_refuses_what_is_not_on_a_gpu():
    x, g = torch.zeros(4, 8), torch.ones(8)
    q, s = x.to(torch.float8_e4m3fn), torch.zeros(4, 1).to(torch.float8_e8m0fnu)
    off = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: agcn.quantize(x), lambda: agcn.quantize(None), lambda: agcn.quantize_weight(x),
                 lambda: agcn.quantize_weight(None), lambda: agcn.rms_norm(x, g),
                 lambda: agcn.rms_norm(None, g), lambda: agcn.quantized_linear(q, s, q, s),
                 lambda: agcn.grouped_linear(q, s, q[None], s[None], off),
                 lambda: agcn.grouped_linear(q, s, q[None], s[None], None),
                 lambda: agcn.grouped_linear(q, s, q[None], s[None], [0, 4])):
        with pytest.raises((TypeError, ValueError)):
            call()
