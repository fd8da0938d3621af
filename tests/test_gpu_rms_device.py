"""Devices with root-mean-square norms, orthogonalised updates and 8-bit uploads
feed the server, and the gradients of the operators as a device chains them agree
with torch's in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2504_13850_gb300 import api, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    api.lib()


def test_devices_feed_the_server():
    from paper_2504_13850_gb300 import sequence
    local, server = sequence.run(events=8, devices=2, vocab=500, kind=sequence.RmsDevice)
    assert len(local) == len(server) == 8 and np.all(np.isfinite(local)) and np.all(np.isfinite(server))


def test_a_step_changes_each_parameter_once():
    """What a step leaves is what the optimisers' definitions give for its
    gradients; the upload decodes to the activations."""
    from paper_2504_13850_gb300 import sequence as S
    d = S.RmsDevice(3, vocab=300, width=128, heads=2, blocks=2, lr=0.05, matrix_lr=0.1, momentum=0.8, weight_decay=0.1)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens, lengths = torch.randint(300, (5, 40), device="cuda", generator=g), torch.tensor([40, 7, 1, 33, 20], device="cuda")
    labels = torch.randint(2, (5,), device="cuda", generator=g)
    y = d.forward(tokens, lengths)[0].detach()
    before, others = [p.detach().clone() for p in d.matrices], [p.detach().clone() for p in d.others]
    (q, scales), loss = d.step(tokens, lengths, labels)
    assert math.isfinite(float(loss)) and q.shape == y.shape
    # an 8-bit value is within 2^-4 of itself or half a step of the group's, and y was rounded to bf16 once more
    step = torch.pow(2.0, scales.double() - 127).repeat_interleave(32, 2)
    off = (api.decode_8bit(q, scales, dtype=torch.float32).double() - y.double()).abs()
    assert bool((off <= (2.0 ** -4 + 2.0 ** -8) * y.double().abs() + 2.0 ** -10 * step).all())
    for p, b, m in zip(d.matrices, before, d.momenta):
        assert torch.equal(m, p.grad)                                   # the first step's momentum
        X = api.orthogonalize(1.8 * p.grad)
        want = b * (1 - 0.1 * 0.1) - 0.1 * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * X
        # X of the same update in another scaling: fp32 roundings that five steps of slope up to 4 pass on
        assert float((p.detach() - want).norm()) <= 1e-4 * 0.1 * float(X.norm()) + 2.0 ** -22 * float(b.norm())
    for p, b in zip(d.others, others):
        assert torch.allclose(p.detach(), b - 0.05 * p.grad, rtol=1e-6, atol=1e-7)
    assert float(d.embedding.grad[tokens[2, 1:]].abs().max()) >= 0      # padding adds nothing:
    seen = torch.zeros(300, dtype=torch.bool, device="cuda")
    for b in range(5):
        seen[tokens[b, :lengths[b]]] = True
    assert bool((d.embedding.grad[~seen] == 0).all())


def test_chain_gradients_match_torch():
    """Embedding, a norm, a product, the norm with the residual's addition, another
    product and the norm of the upload, as the device chains them, against the same
    chain in 64 bits.  Bound: each of the nine bf16 tensors on the way (x, h, both
    branches, s twice, y and their gradients' chain) is off by 2^-8 relative per
    element, and so are the two rounded weights; errors of independent elements add
    in the 2-norm, so 11 * 2^-8 covers every gradient normwise."""
    from paper_2504_13850_gb300 import sequence as S
    T, V, D = 300, 50, 160
    g = torch.Generator(device="cuda").manual_seed(5)

    def leaf(*shape, scale=1.0, shift=0.0):
        return (shift + scale * torch.randn(*shape, device="cuda", generator=g)).requires_grad_()

    table, a, b = leaf(V, D), leaf(D, D, scale=D ** -0.5), leaf(D, D, scale=D ** -0.5)
    w = [leaf(D, scale=0.2, shift=1.0) for _ in range(3)]
    ids = torch.randint(-1, V, (T,), device="cuda", generator=g)
    dy = torch.randn(T, D, device="cuda", generator=g).bfloat16()
    linear = torch.nn.functional.linear
    x = S.TokenEmbedding.apply(table, ids, 1.5)
    h = S.Norm.apply(x, w[0])
    h, s = S.AddNorm.apply(linear(h, a.bfloat16()), x, w[1])
    y, q, scales = S.UploadNorm.apply(linear(h, b.bfloat16()), s, w[2])
    y.backward(dy)

    ref = [t.detach().double().requires_grad_() for t in (table, a, b, *w)]

    def norm(t, weight):
        return t * (t.square().mean(1, keepdim=True) + 1e-6) ** -0.5 * weight

    X = torch.where((ids >= 0)[:, None], ref[0][ids.clamp(min=0)] * 1.5, 0.0)
    s1 = linear(norm(X, ref[3]), ref[1]) + X
    Y = norm(linear(norm(s1, ref[4]), ref[2]) + s1, ref[5])
    Y.backward(dy.double())
    for name, got, want in zip(("y", "table", "a", "b", "w0", "w1", "w2"), (y, *(t.grad for t in (table, a, b, *w))),
                               (Y, *(t.grad for t in ref))):
        err = float((got.detach().double() - want.detach()).norm() / want.detach().norm())
        assert err <= 11 * 2.0 ** -8, (name, err)


def test_backward_in_a_graph_beside_an_eager_one():
    """A forward and backward pass of the functions captured and replayed while an
    eager graph of other leaves is alive."""
    from paper_2504_13850_gb300 import sequence as S
    table, w = torch.randn(30, 64, device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True)
    ids = torch.randint(30, (100,), device="cuda")

    def loss(table, w):
        x = S.TokenEmbedding.apply(table, ids, 1.0)
        y, s = S.AddNorm.apply(x, x, w)
        return (y.float() * s.float()).sum()

    eager = [t.detach().clone().requires_grad_() for t in (table, w)]
    alive = loss(*eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(loss(table, w), (table, w))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = torch.autograd.grad(loss(table, w), (table, w))
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(grads, torch.autograd.grad(alive, eager)):
        assert torch.equal(a, b)
