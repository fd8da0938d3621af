"""The host side of embedding and norm, without a GPU: refusals of the C ABI and
workspace sizes, and of the compiled binding."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


P = 4096                                # an address that no refused call reads


def embedding(**over):
    a = dict(ids=P, bits=32, tokens=4, table=P, table_dtype=0, vocab=10, width=8, scale=1.0, out=P, stride=8, dtype=0)
    a.update(over)
    return api.lib().fo_embedding(*a.values(), None)


def embedding_grad(**over):
    a = dict(dout=P, stride=8, dtype=0, ids=P, bits=32, tokens=4, dtable=P, table_dtype=0, vocab=10, width=8, scale=1.0, accumulate=0,
             workspace=P, bytes=1 << 30)
    a.update(over)
    return api.lib().fo_embedding_grad(*a.values(), None)


SIZES = [({"bits": 16}, "bits"), ({"tokens": -1}, "tokens"), ({"tokens": (1 << 30) + 1}, "tokens"), ({"vocab": 0}, "rows"),
         ({"vocab": (1 << 30) + 1}, "rows"), ({"width": 0}, "columns"), ({"width": (1 << 20) + 1}, "columns"), ({"dtype": 2}, "fp32"),
         ({"table_dtype": 5}, "fp32"), ({"table_dtype": 1}, "fp32 table"), ({"ids": None}, "pointer"), ({"ids": P + 2}, "pointer"),
         ({"bits": 64, "ids": P + 4}, "pointer")]


@pytest.mark.parametrize("over,what", SIZES + [({"table": None}, "pointer"), ({"out": P + 1}, "pointer"), ({"stride": 7}, "stride"),
                                               ({"stride": 1 << 62}, "stride")])
def test_bad_lookups_are_refused(over, what):
    assert embedding(**over) == api.ERR_ARG and what in api.last_error()


@pytest.mark.parametrize("over,what", SIZES + [({"dtable": None}, "dtable"), ({"dout": None}, "pointer"), ({"stride": -1}, "stride"),
                                               ({"workspace": None}, "workspace"), ({"workspace": P + 16}, "workspace"),
                                               ({"bytes": 100}, "workspace")])
def test_bad_embedding_gradients_are_refused(over, what):
    assert embedding_grad(**over) == api.ERR_ARG and what in api.last_error()


def norm(**over):
    a = dict(x=P, xs=8, residual=None, rs=0, weight=P, weight_dtype=0, sum=None, ss=0, y=P + 4096, ys=8, q=None, scales=None, rstd=None,
             dtype=0, rows=4, cols=8, eps=1e-6)
    a.update(over)
    return api.lib().fo_rms_norm(*a.values(), None)


def norm_grad(**over):
    a = dict(dy=P, dys=8, ds=None, dss=0, s=P, ss=8, weight=P, weight_dtype=0, rstd=P, dx=P, dxs=8, dweight=P, dtype=0, rows=4, cols=8,
             workspace=P, bytes=1 << 30)
    a.update(over)
    return api.lib().fo_rms_norm_grad(*a.values(), None)


@pytest.mark.parametrize("over,what", [
    ({"dtype": 2}, "dtype"), ({"rows": -1}, "rows"), ({"rows": 1 << 31}, "rows"), ({"cols": 0}, "columns"),
    ({"cols": (1 << 20) + 1}, "columns"), ({"weight_dtype": 1}, "weight"), ({"weight": None}, "weight"), ({"x": None}, "x is"),
    ({"x": P + 2}, "x is"), ({"xs": -1}, "stride of x"), ({"ys": 7}, "stride of y"), ({"eps": -1e-9}, "eps"), ({"eps": float("inf")}, "eps"),
    ({"y": None}, "neither"), ({"q": P}, "together"), ({"scales": P}, "together"), ({"residual": P, "rs": 8}, "sum"),
    ({"residual": P, "rs": 8, "sum": P + 4096, "ss": 8}, "one tensor"), ({"rstd": P + 2}, "rstd"),
    ({"residual": P, "rs": 8, "sum": P, "ss": 4}, "stride of sum")])
def test_bad_norms_are_refused(over, what):
    assert norm(**over) == api.ERR_ARG and what in api.last_error()


@pytest.mark.parametrize("over,what", [
    ({"dtype": 3}, "dtype"), ({"cols": 0}, "columns"), ({"weight_dtype": 1}, "weight"), ({"dweight": None}, "dweight"),
    ({"dy": None}, "dy"), ({"s": P + 1}, "s is"), ({"dx": None}, "dx"), ({"rstd": None}, "rstd"), ({"dxs": 7}, "stride of dx"),
    ({"ds": P, "dss": -8}, "stride of ds"), ({"workspace": None}, "workspace"), ({"workspace": P + 8}, "workspace"), ({"bytes": 31}, "workspace")])
def test_bad_norm_gradients_are_refused(over, what):
    assert norm_grad(**over) == api.ERR_ARG and what in api.last_error()


@pytest.mark.parametrize("args,what", [((None, P, P, 8, 0, 4, 8), "null"), ((P, None, P, 8, 0, 4, 8), "null"), ((P, P, None, 8, 0, 4, 8), "y is"),
                                       ((P, P, P, 7, 0, 4, 8), "stride"), ((P, P, P, 8, 2, 4, 8), "dtype"), ((P, P, P, 8, 0, 4, 0), "columns")])
def test_bad_decodings_are_refused(args, what):
    assert api.lib().fo_decode_8bit(*args, None) == api.ERR_ARG and what in api.last_error()


def test_workspaces():
    L = api.lib()
    assert L.fo_embedding_workspace(0, 8) == 0 and L.fo_embedding_workspace(-1, 8) == -1 and L.fo_embedding_workspace(8, 0) == -1
    sizes = [L.fo_embedding_workspace(t, 512) for t in (1, 100, 10000, 1000000)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert L.fo_rms_norm_workspace(0, 8) == 0 and L.fo_rms_norm_workspace(1, 0) == -1 and L.fo_rms_norm_workspace(1 << 31, 8) == -1
    assert L.fo_rms_norm_workspace(1, 100) >= 400


def test_the_compiled_binding_refuses_what_is_no_device_tensor():
    """Checks that come before any call of the library."""
    x, ids, w = torch.ones(2, 4), torch.zeros(2, dtype=torch.int32), torch.ones(4)
    q = torch.zeros(2, 4, dtype=torch.uint8).view(torch.float8_e4m3fn)
    for call in (lambda: api.embedding(ids, x), lambda: api.embedding_grad(x, ids, 3), lambda: api.rms_norm(x, None, w),
                 lambda: api.rms_norm(x.half(), None, w), lambda: api.rms_norm_8bit(x, None, w), lambda: api.rms_norm_grad(x, None, x, w, w),
                 lambda: api.decode_8bit(q, ids), lambda: api.orthogonalize(x), lambda: api.orthogonalize([x], out=[x, x]),
                 lambda: api.orthogonalize([x], coefficients=(1.0, 2.0)), lambda: api.muon_step([x], [x, x], [x], 0.1),
                 lambda: api.muon_step([x], [x], [x], 0.1, scales=[1.0, 2.0])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: api.embedding(3, x), lambda: api.rms_norm("x", None, w), lambda: api.orthogonalize([1.0]),
                 lambda: api.orthogonalize([x], steps="5", eps=None)):
        with pytest.raises((TypeError, ValueError)):
            call()
    assert api.orthogonalize([]) == [] and api.muon_step([], [], [], 0.1) is None


def test_matrix_updates_have_the_headers_layout():
    import ctypes as C
    assert C.sizeof(api.fo_matrix_update) == 88 and api.fo_matrix_update.grad.offset == 16 and api.fo_matrix_update.step.offset == 80


def items(*sizes, **over):
    a = (api.fo_matrix_update * len(sizes))()
    for it, (r, c) in zip(a, sizes):
        it.rows, it.cols, it.grad, it.out, it.grad_stride, it.out_stride = r, c, P, P, c, c
        for k, v in over.items():
            setattr(it, k, v)
    return a


def orthogonalize(a, **over):
    import ctypes as C
    k = dict(dtype=0, steps=5, coefficients=(C.c_double * 3)(3.0, -4.0, 2.0), eps=1e-7, mu=0.9, nesterov=1, decay=1.0, workspace=P, bytes=1 << 40)
    k.update(over)
    return api.lib().fo_orthogonalize(a, len(a), *k.values(), None)


@pytest.mark.parametrize("sizes,over,what", [
    ([(-1, 4)], {}, "sides"), ([(32769, 32769)], {}, "sides"), ([(4, (1 << 20) + 1)], {}, "sides"),
    ([(4, 4)], {"grad": None}, "pointer"), ([(4, 4)], {"grad": P + 2}, "pointer"), ([(4, 4)], {"momentum": P + 2}, "pointer"),
    ([(4, 4)], {"out": None}, "neither"), ([(4, 4)], {"out_stride": 3}, "stride"), ([(4, 4)], {"grad_stride": -1}, "stride"),
    ([(4, 4)], {"param": P, "param_stride": 2}, "stride"), ([(4, 4)], {"step": float("nan")}, "step")])
def test_bad_matrices_are_refused(sizes, over, what):
    assert orthogonalize(items(*sizes, **over)) == api.ERR_ARG and what in api.last_error()


@pytest.mark.parametrize("field", ["out", "momentum", "param"])
def test_a_tensor_to_write_twice_is_refused(field):
    a = items((4, 4), (4, 4), out_stride=4, momentum_stride=4, param_stride=4)
    for k, it in enumerate(a):
        it.out, it.momentum, it.param = P + 4096 * k, P + 65536 * (1 + k), P + 1048576 * (1 + k)
    setattr(a[1], field, getattr(a[0], field))
    assert orthogonalize(a) == api.ERR_ARG and "twice" in api.last_error()


@pytest.mark.parametrize("to,name,what", [(39, "out", 0), (39, "grad", 0), (0, "grad", 39), (5, "momentum", 5), (7, "param", 7), (7, "param", 30)])
def test_tensors_written_by_another_place_of_the_list_are_refused(to, name, what):
    """out of matrix `what` as `name` of matrix `to`, launches apart or the same; a
    matrix's own grad may be its out."""
    a = items(*[(4, 4)] * 40, out_stride=4, momentum_stride=4, param_stride=4)
    for k, it in enumerate(a):
        it.grad, it.out, it.momentum, it.param = (P + 4096 * (4 * k + j) for j in range(4))
    assert orthogonalize(a, workspace=None) == api.ERR_ARG and "workspace" in api.last_error()
    a[3].out = a[3].grad
    assert orthogonalize(a, workspace=None) == api.ERR_ARG and "workspace" in api.last_error()
    setattr(a[to], name, a[what].out)
    assert orthogonalize(a, workspace=None) == api.ERR_ARG and "twice" in api.last_error()


@pytest.mark.parametrize("over,what", [
    ({"dtype": 2}, "dtype"), ({"steps": 0}, "steps"), ({"steps": 65}, "steps"), ({"coefficients": None}, "coefficients"), ({"eps": 0.0}, "eps"),
    ({"mu": -0.1}, "momentum"), ({"mu": float("nan")}, "momentum"), ({"decay": float("inf")}, "decay"), ({"workspace": None}, "workspace"),
    ({"workspace": P + 8}, "workspace"), ({"bytes": 1000}, "workspace")])
def test_bad_orthogonalisations_are_refused(over, what):
    assert orthogonalize(items((200, 300)), **over) == api.ERR_ARG and what in api.last_error()


def test_orthogonalize_workspaces():
    L = api.lib()
    assert L.fo_orthogonalize_workspace(items((0, 5), (5, 0)), 2, 0) == 0 and L.fo_orthogonalize_workspace(None, 0, 0) == 0
    assert L.fo_orthogonalize_workspace(None, 1, 0) == -1 and L.fo_orthogonalize_workspace(items((1, 1)), 1, 7) == -1
    one = L.fo_orthogonalize_workspace(items((512, 700)), 1, 0)
    assert one >= 8 * (512 * 700 + 512 * 512) and L.fo_orthogonalize_workspace(items(*[(512, 700)] * 40), 40, 0) == 32 * one
