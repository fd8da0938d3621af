"""An optimiser step's parameters are fp32, and the orthogonalised update that reaches
them is as exact for bf16 gradients as for fp32 ones."""
import pytest
import torch

from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()
    yield
    api.orthogonalize_error()


def exact(u, steps=5):
    a, b, c = api.QUINTIC
    x = u.double() if u.shape[0] <= u.shape[1] else u.double().t()
    x = x / (x.norm() + 1e-7)
    for _ in range(steps):
        A = x @ x.t()
        x = a * x + (b * A + c * A @ A) @ x
    return x if u.shape[0] <= u.shape[1] else x.t()


SHAPES = [(512, 768), (90, 150), (300, 128), (256, 256), (140, 2100)]


@pytest.mark.parametrize("dtype", [F32, BF])
def test_updates_of_parameters(dtype):
    """Singular values of a random matrix grow as their errors do, or end where an error passes on with a slope of
    at most 4; products and storage lose fewer than 16 * 2^-23 of their size in each of the five steps."""
    params = [torch.zeros(s, device="cuda") for s in SHAPES]
    grads = [torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k)).to(dtype) for k, s in enumerate(SHAPES)]
    api.muon_step(params, grads, [torch.zeros_like(p) for p in params], 1.0, momentum=0.0, scales=[1.0] * len(SHAPES))
    for p, g in zip(params, grads):
        want = -exact(g)
        assert float((p.double() - want).norm()) <= 5 * 16 * 2.0 ** -23 * 4 * float(want.norm())


def test_outputs_and_parameters_of_one_list():
    """A list with bf16 matrices that update parameters, ones that only have an output, and small ones of both
    kinds: each as it is alone."""
    import ctypes as C
    shapes = [(200, 300), (300, 200), (64, 90), (90, 64), (700, 130)]
    grads = [torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k)).to(BF) for k, s in enumerate(shapes)]

    def call(which):
        items = (api.fo_matrix_update * len(which))()
        outs, params = {}, {}
        for it, k in zip(items, which):
            r, c = shapes[k]
            it.rows, it.cols, it.grad, it.grad_stride, it.step = r, c, grads[k].data_ptr(), c, 1.0
            if k % 2:
                params[k] = torch.zeros(r, c, device="cuda")
                it.param, it.param_stride = params[k].data_ptr(), c
            if k != 3:
                outs[k] = torch.empty(r, c, device="cuda", dtype=BF)
                it.out, it.out_stride = outs[k].data_ptr(), c
        need = api.lib().fo_orthogonalize_workspace(items, len(which), 1)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        rc = api.lib().fo_orthogonalize(items, len(which), 1, 5, (C.c_double * 3)(*api.QUINTIC), 1e-7, 0.0, 0, 1.0, ws.data_ptr(), need,
                                        torch.cuda.current_stream().cuda_stream)
        assert rc == 0, api.last_error()
        torch.cuda.synchronize()
        return outs, params

    outs, params = call(range(5))
    for k in range(5):
        o, p = call([k])
        assert k not in o or torch.equal(o[k], outs[k])
        assert k not in p or torch.equal(p[k], params[k])
        if k in p and k in o:
            assert torch.equal(o[k], (-p[k]).to(BF))
