"""The host side of embedding and norm, without a GPU: refusals of the C ABI and
workspace sizes, and the tensors' device made current by the binding."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build
from test_operators_device import Machine, Tensor


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


class Stand(Machine):
    def __init__(self, monkeypatch):
        super().__init__(monkeypatch)
        api._setup(torch)
        monkeypatch.setattr(api, "_raw_stream", lambda index: 0)

    def fo_embedding_workspace(self, tokens, width):
        return 256

    def fo_rms_norm_workspace(self, rows, cols):
        return 256

    def fo_orthogonalize_workspace(self, items, count, dtype):
        return 256


def ids(index):
    return Tensor((2, 16), torch.int32, index)


def matrix(index, dtype=torch.bfloat16):
    return Tensor((2, 16, 64), dtype, index)


def vector(index):
    return Tensor((64,), torch.float32, index)


def codes(index):
    return Tensor((2, 16, 64), torch.float8_e4m3fn, index), Tensor((2, 16, 2), torch.uint8, index)


CALLS = {
    "fo_embedding": lambda i, **kw: api.embedding(ids(i), Tensor((10, 64), torch.float32, i), dtype=torch.bfloat16, **kw),
    "fo_embedding_grad": lambda i, **kw: api.embedding_grad(matrix(i), ids(i), 10, dtype=torch.float32, **kw),
    "fo_rms_norm": lambda i, **kw: api.rms_norm(matrix(i), matrix(i), vector(i), **kw),
    "fo_rms_norm_grad": lambda i, **kw: api.rms_norm_grad(matrix(i), matrix(i), matrix(i), vector(i), Tensor((2, 16), torch.float32, i), **kw),
    "fo_decode_8bit": lambda i, **kw: api.decode_8bit(*codes(i), **kw),
    "fo_orthogonalize": lambda i, **kw: api.orthogonalize([Tensor((9, 5), torch.float32, i)] * 2, **kw),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("index", [0, 1])
@pytest.mark.parametrize("stream", [None, 77])
def test_the_tensors_device_is_current(monkeypatch, name, index, stream):
    machine = Stand(monkeypatch)
    CALLS[name](index, stream=stream)
    assert machine.calls == [(name, index, stream or 0)]
    assert set(machine.allocated) == {index} and machine.current == 0


def test_mixed_devices_are_refused(monkeypatch):
    machine = Stand(monkeypatch)
    for call in (lambda: api.embedding(ids(0), Tensor((10, 64), torch.float32, 1)), lambda: api.embedding_grad(matrix(1), ids(0), 10),
                 lambda: api.rms_norm(matrix(0), matrix(1), vector(0)), lambda: api.rms_norm(matrix(0), None, vector(1)),
                 lambda: api.rms_norm_grad(matrix(1), None, matrix(0), vector(0), Tensor((2, 16), torch.float32, 0)),
                 lambda: api.decode_8bit(codes(0)[0], codes(1)[1]),
                 lambda: api.orthogonalize([Tensor((9, 5), torch.float32, i) for i in (0, 1)])):
        with pytest.raises(ValueError):
            call()
    assert machine.calls == [] and machine.current == 0


def test_matrix_updates_are_laid_out_as_the_library_reads_them(monkeypatch):
    """The binding fills the items as 64-bit words."""
    import ctypes as C
    machine, seen = Stand(monkeypatch), []

    def call(items, n, *rest):
        seen.extend((api.fo_matrix_update * n).from_address(items))
        machine.copy = [{f: getattr(m, f) for f, _ in m._fields_} for m in seen]
        return api.OK

    monkeypatch.setattr(Stand, "fo_orthogonalize", staticmethod(call), raising=False)
    shapes = [(9, 5), (7, 30)]
    p, g, m = ([Tensor(s, torch.float32, 0) for s in shapes] for _ in range(3))
    api.muon_step(p, g, m, lr=0.5, scales=[3.0, -0.25])
    assert C.sizeof(api.fo_matrix_update) == 88
    for got, (rows, cols), step in zip(machine.copy, shapes, (1.5, -0.125)):
        assert got == dict(rows=rows, cols=cols, grad=4096, momentum=4096, out=None, param=4096, grad_stride=cols, momentum_stride=cols,
                           out_stride=0, param_stride=cols, step=step)
    for bad in (lambda: api.muon_step(p, g[:1], m, 0.1), lambda: api.muon_step(p, g, m, 0.1, scales=[1.0]),
                lambda: api.orthogonalize(g, coefficients=(1.0, 2.0))):
        with pytest.raises(ValueError):
            bad()


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
