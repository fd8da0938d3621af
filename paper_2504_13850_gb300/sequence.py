"""Devices that train transformer blocks beside the server, in two kinds.

The transformer workload's server trains blocks behind the split (Sec. 3.2); the
part in front of it, M_dk (an embedding and two blocks, as the workload counts
them), with its auxiliary head trains here on the device, with the operators that the server's network does not have: attention with a learned
relative position bias over padded batches (``api.attention_forward`` /
``attention_backward``) and dropout around the residuals
(``api.dropout_add`` / ``dropout_grad``).  Products, layer norms and the GELU are
torch's.  One event follows Algorithm 1: a local iteration with the local loss
f_d, then the upload of its split-point activations, which the server trains on
(Algorithms 2 and 3).

``RmsDevice`` trains blocks of another kind: a scaled token embedding
(``api.embedding`` / ``embedding_grad``), root-mean-square norms that take the
residual's addition with them (``api.rms_norm`` / ``rms_norm_grad``), and weight
matrices whose momentum is made orthogonal before each step
(``api.muon_step``).  It hands over its split-point activations in 8 bits
(``api.rms_norm_8bit``), a form of half the bytes S_l / b_k of Eq. 5 that bf16
takes.  Here the devices share the server's GPU and no link is crossed:
``run`` decodes them beside the server (``api.decode_8bit``), whose slots take
bf16.

    python -m paper_2504_13850_gb300.sequence [--rms]
"""
import sys

import torch
from torch.autograd.function import once_differentiable

from . import api
from . import workloads as W

BUCKETS, REACH = 32, 128


class PackedAttention(torch.autograd.Function):
    """o [B, L, H, D] of one projection qkv [B, L, 3, H, D]; the three gradients
    are written into one gradient of the projection."""

    @staticmethod
    def forward(ctx, qkv, table, buckets, documents):
        q, k, v = qkv.unbind(2)
        o, lse = api.attention_forward(q, k, v, table=table, buckets=buckets, documents=documents)
        ctx.save_for_backward(qkv, table, documents, o, lse)
        ctx.buckets = buckets
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        qkv, table, documents, o, lse = ctx.saved_tensors
        q, k, v = qkv.unbind(2)
        dqkv = torch.empty_like(qkv)
        *_, dtable = api.attention_backward(do, q, k, v, o, lse, table=table, buckets=ctx.buckets, documents=documents,
                                            grads=dqkv.unbind(2))
        return dqkv, dtable, None, None


class ResidualDropout(torch.autograd.Function):
    """residual + dropout(x); the mask is drawn again in the backward pass."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, call):
        ctx.mask = p, seed, call
        return api.dropout_add(x, residual, p, seed, call)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        dy = dy.contiguous()
        return api.dropout_grad(dy, *ctx.mask), dy, None, None, None


class SequenceDevice:
    """One device: embedding, pre-LN blocks, auxiliary head; bf16 compute on
    fp32 parameters, SGD with momentum."""

    def __init__(self, seed, vocab=30522, width=512, heads=8, blocks=2, classes=2, p=0.1, lr=0.01, momentum=0.9):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.width, self.heads, self.p, self.seed, self.steps = width, heads, p, seed, 0
        self.buckets = api.relative_buckets(BUCKETS, REACH)

        def weight(n, m):
            return (torch.randn(n, m, device="cuda", generator=g) * m ** -0.5).requires_grad_()

        def vector(n, value=0.0):
            return torch.full((n,), value, device="cuda").requires_grad_()

        self.embedding = torch.randn(vocab, width, device="cuda", generator=g).requires_grad_()
        self.blocks = [{"ln1": vector(width, 1.0), "ln1_b": vector(width), "qkv": weight(3 * width, width),
                        "table": torch.zeros(heads, BUCKETS, device="cuda").requires_grad_(),
                        "proj": weight(width, width), "ln2": vector(width, 1.0), "ln2_b": vector(width),
                        "up": weight(4 * width, width), "down": weight(width, 4 * width)} for _ in range(blocks)]
        self.head = weight(classes, width)
        self.params = [self.embedding, self.head] + [t for b in self.blocks for t in b.values()]
        self.opt = torch.optim.SGD(self.params, lr=lr, momentum=momentum)

    def forward(self, tokens, lengths):
        """Split-point activations [B, L, width] (bf16) of tokens [B, L]."""
        B, L = tokens.shape
        # tokens past a sequence's length are padding: in no document
        documents = torch.where(torch.arange(L, device=tokens.device) < lengths[:, None], 0, -1).to(torch.int32)
        norm, linear = torch.nn.functional.layer_norm, torch.nn.functional.linear
        x = self.embedding[tokens].bfloat16()
        for i, b in enumerate(self.blocks):
            w = {n: t.bfloat16() for n, t in b.items()}
            call = self.steps * 2 * len(self.blocks) + 2 * i          # another mask for each use
            qkv = linear(norm(x, (self.width,), w["ln1"], w["ln1_b"]), w["qkv"])
            o = PackedAttention.apply(qkv.view(B, L, 3, self.heads, -1), w["table"], self.buckets, documents)
            x = ResidualDropout.apply(linear(o.reshape(B, L, -1), w["proj"]), x, self.p, self.seed, call)
            h = torch.nn.functional.gelu(linear(norm(x, (self.width,), w["ln2"], w["ln2_b"]), w["up"]))
            x = ResidualDropout.apply(linear(h, w["down"]), x, self.p, self.seed, call + 1)
        return x

    def step(self, tokens, lengths, labels):
        """One local iteration with the auxiliary head's loss f_d (softmax
        cross-entropy of the mean over valid tokens): (activations, loss)."""
        self.opt.zero_grad(set_to_none=True)
        x = self.forward(tokens, lengths)
        valid = (torch.arange(tokens.shape[1], device=tokens.device) < lengths[:, None]).unsqueeze(2)
        pooled = (x.float() * valid).sum(1) / lengths[:, None]
        loss = torch.nn.functional.cross_entropy(pooled @ self.head.t(), labels.long())
        loss.backward()
        # waits for the step's work, so that x may be uploaded from another
        # stream; a kernel that gave up a wait ends the step before it changes
        # a parameter
        api.attention_error()
        self.opt.step()
        self.steps += 1
        return x.detach(), loss.detach()


class TokenEmbedding(torch.autograd.Function):
    """scale * table[ids] in bf16, of an fp32 table; zeros for padding (ids < 0)."""

    @staticmethod
    def forward(ctx, table, ids, scale):
        ctx.save_for_backward(ids)
        ctx.how = table.shape[0], scale
        return api.embedding(ids, table, scale=scale, dtype=torch.bfloat16)

    @staticmethod
    @once_differentiable
    def backward(ctx, dx):
        vocab, scale = ctx.how
        return api.embedding_grad(dx, *ctx.saved_tensors, vocab, scale=scale, dtype=torch.float32), None, None


class Norm(torch.autograd.Function):
    """Root-mean-square norm of x."""

    @staticmethod
    def forward(ctx, x, weight):
        y, _, r = api.rms_norm(x, None, weight)
        ctx.save_for_backward(x, weight, r)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, r = ctx.saved_tensors
        return api.rms_norm_grad(dy, None, x, weight, r)


class AddNorm(torch.autograd.Function):
    """(norm of x + residual, x + residual)."""

    @staticmethod
    def forward(ctx, x, residual, weight):
        y, s, r = api.rms_norm(x, residual, weight)
        ctx.save_for_backward(s, weight, r)
        return y, s

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds):
        dx, dw = api.rms_norm_grad(dy, ds, *ctx.saved_tensors)
        return dx, dx, dw


class UploadNorm(torch.autograd.Function):
    """The norm of x + residual and its 8-bit form (values, scales), which has no
    gradient."""

    @staticmethod
    def forward(ctx, x, residual, weight):
        q, scales, y, s, r = api.rms_norm_8bit(x, residual, weight, with_y=True)
        ctx.save_for_backward(s, weight, r)
        ctx.mark_non_differentiable(q, scales)
        return y, q, scales

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, *_):
        s, weight, r = ctx.saved_tensors
        dx, dw = api.rms_norm_grad(dy, None, s, weight, r)
        return dx, dx, dw


class RmsDevice:
    """One device with root-mean-square norms and orthogonalised updates; bf16
    compute on fp32 parameters.  The embedding, norms, bias tables and head are
    trained by SGD with momentum."""

    def __init__(self, seed, vocab=30522, width=512, heads=8, blocks=2, classes=2, lr=0.01, matrix_lr=0.02, momentum=0.9,
                 weight_decay=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.width, self.heads, self.buckets = width, heads, api.relative_buckets(BUCKETS, REACH)
        self.matrix_lr, self.momentum, self.weight_decay = matrix_lr, momentum, weight_decay

        def matrix(n, m):
            return (torch.randn(n, m, device="cuda", generator=g) * m ** -0.5).requires_grad_()

        def ones():
            return torch.ones(width, device="cuda").requires_grad_()

        self.embedding = (torch.randn(vocab, width, device="cuda", generator=g) * width ** -0.5).requires_grad_()
        self.blocks = [{"norm1": ones(), "qkv": matrix(3 * width, width),
                        "table": torch.zeros(heads, BUCKETS, device="cuda").requires_grad_(), "proj": matrix(width, width),
                        "norm2": ones(), "up": matrix(4 * width, width), "down": matrix(width, 4 * width)} for _ in range(blocks)]
        self.norm, self.head = ones(), matrix(classes, width)
        self.matrices = [b[n] for b in self.blocks for n in ("qkv", "proj", "up", "down")]
        self.momenta = [torch.zeros_like(m) for m in self.matrices]
        self.others = [self.embedding, self.norm, self.head] + [b[n] for b in self.blocks for n in ("norm1", "table", "norm2")]
        self.opt = torch.optim.SGD(self.others, lr=lr, momentum=momentum)

    def forward(self, tokens, lengths):
        """Split-point activations [B, L, width] (bf16) of tokens [B, L], and their 8-bit form."""
        B, L = tokens.shape
        valid = torch.arange(L, device=tokens.device) < lengths[:, None]
        documents = torch.where(valid, 0, -1).to(torch.int32)
        linear = torch.nn.functional.linear
        x = TokenEmbedding.apply(self.embedding, torch.where(valid, tokens, -1), self.width ** 0.5)
        branch = None
        for b in self.blocks:
            w = {n: b[n].bfloat16() for n in ("qkv", "table", "proj", "up", "down")}
            h, x = (Norm.apply(x, b["norm1"]), x) if branch is None else AddNorm.apply(branch, x, b["norm1"])
            o = PackedAttention.apply(linear(h, w["qkv"]).view(B, L, 3, self.heads, -1), w["table"], self.buckets, documents)
            h, x = AddNorm.apply(linear(o.reshape(B, L, -1), w["proj"]), x, b["norm2"])
            branch = linear(torch.nn.functional.gelu(linear(h, w["up"])), w["down"])
        return UploadNorm.apply(branch, x, self.norm)

    def step(self, tokens, lengths, labels):
        """One local iteration with the auxiliary head's loss f_d (softmax
        cross-entropy of the mean over valid tokens): ((8-bit activations, their
        scales), loss)."""
        for p in self.matrices:
            p.grad = None
        self.opt.zero_grad(set_to_none=True)
        x, *upload = self.forward(tokens, lengths)
        valid = (torch.arange(tokens.shape[1], device=tokens.device) < lengths[:, None]).unsqueeze(2)
        pooled = (x.float() * valid).sum(1) / lengths[:, None]
        loss = torch.nn.functional.cross_entropy(pooled @ self.head.t(), labels.long())
        loss.backward()
        # waits for the step's work; a kernel that gave up a wait ends the step
        # before it changes a parameter
        api.attention_error()
        changed = [t.detach() for t in (*self.matrices, *self.momenta)]
        before = [t.clone() for t in changed]
        try:
            api.muon_step(self.matrices, [p.grad for p in self.matrices], self.momenta, self.matrix_lr, momentum=self.momentum,
                          weight_decay=self.weight_decay)
            api.orthogonalize_error()
        except api.FedOptimaError:             # part of them is void
            for t, b in zip(changed, before):
                t.copy_(b)
            raise
        self.opt.step()
        return tuple(t.detach() for t in upload), loss.detach()


def run(events=32, devices=4, seed=0, vocab=30522, kind=SequenceDevice):
    """Device events and server iterations; returns the local and server losses."""
    cfg = dict(W.CONFIGS["transformer"], K=devices, omega=4 * devices)
    B, L = cfg["batch"], cfg["in_hwc"][0]
    server = api.Server.from_config(cfg)
    server.set_params(W.init_params(cfg))
    g = torch.Generator(device="cuda").manual_seed(seed)
    parts = [kind(seed + k, vocab) for k in range(devices)]
    data = [(torch.randint(vocab, (B, L), device="cuda", generator=g),
             torch.randint(32, L + 1, (B,), device="cuda", generator=g, dtype=torch.int32),
             torch.randint(2, (B,), device="cuda", generator=g, dtype=torch.int32)) for _ in range(devices)]
    local = []
    for e in range(events):
        k = e % devices
        tokens, lengths, labels = data[k]
        x, loss = parts[k].step(tokens, lengths, labels)
        local.append(loss)
        if kind is RmsDevice:                  # what arrived, for the server's slot
            x = api.decode_8bit(*x)
            torch.cuda.current_stream().synchronize()
        if server.enqueue_activations(k, x, labels, lengths)[0] == api.OK:
            server.server_step()
    server.synchronize()
    server.check_error()
    losses = server.read_losses(0, events)
    server.close()
    return torch.stack(local).tolist(), losses.tolist()


if __name__ == "__main__":
    local, global_ = run(kind=RmsDevice if "--rms" in sys.argv[1:] else SequenceDevice)
    print("device losses", [round(v, 3) for v in local])
    print("server losses", [round(v, 3) for v in global_])
