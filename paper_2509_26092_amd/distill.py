"""Distillation from a trained network: the teacher's top logits are kept once
a batch, and a student learns from them and the labels.

Two students: the library's own ResNet-18 step (Worker.train_step_distill),
and TokenStudent, a small network of patches with layer norm over channels and,
where asked for, residual blocks that mix the patches by linear attention. Its
forward and backward passes call the library's operators (its products, ReLU
and means are torch's, as in a network of the user's).

    python -m paper_2509_26092_amd.distill --student tokens --steps 50
    python -m paper_2509_26092_amd.distill --student tokens --blocks 2 --dropout 0.1
"""
import argparse

import torch

from . import binding as B
from . import inputs

EPS = 1e-5


def _prec(t):
    return {torch.float32: B.RN18_FP32, torch.bfloat16: B.RN18_BF16, torch.float16: B.RN18_FP16}[t.dtype]


def teacher_targets(worker, state, images, k):
    """(values, classes) [N][k] of the teacher's largest logits for a batch.
    All of it runs on the worker's stream, after what is on the current one
    (the images, the state); the current stream waits for the result."""
    n, c = images.shape[0], worker.cfg.num_classes
    here = torch.cuda.current_stream()
    worker.stream.wait_stream(here)
    with torch.cuda.stream(worker.stream):
        logits = torch.empty((n, c), device="cuda")
        worker.eval_logits(state, images, logits)
        vals = torch.empty((n, k), device="cuda")
        idx = torch.empty((n, k), dtype=torch.int32, device="cuda")
        need = B.rn18op_topk_logits_workspace(B.RN18_FP32, n, c, k)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        B.rn18op_topk_logits(B.RN18_FP32, logits, vals, idx, n, c, logits.stride(0), k, ws)
    here.wait_stream(worker.stream)
    for t in (vals, idx):           # made on the worker's stream, read on the current one
        t.record_stream(here)
    return vals, idx


def _rows(t):
    """`t` [rows][width] and its row stride: as it is where the elements of a
    row are one after the other and rows do not overlap, otherwise a copy."""
    r, d = t.shape
    if (d > 1 and t.stride(1) != 1) or (r > 1 and t.stride(0) < d):
        t = t.contiguous()
    return t, t.stride(0) if r > 1 else d


def _workspace(need):
    """Scratch of one call: no other stream's, and of a captured call its graph's own."""
    return torch.empty(need, dtype=torch.uint8, device="cuda") if need else None


class LayerNorm:
    """Layer norm over the last axis of [rows][width]: parameters, what the
    backward pass needs, and gradients."""

    def __init__(self, width):
        self.gamma, self.beta = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)

    def forward(self, x):
        r, d = x.shape
        if d != len(self.gamma):
            raise ValueError("rows of %d elements for a layer norm of %d" % (d, len(self.gamma)))
        self.prec = _prec(x)
        self.x, self.ldx = _rows(x)
        y = torch.empty((r, d), dtype=x.dtype, device=x.device)
        self.mean, self.rstd = torch.empty(r, device="cuda"), torch.empty(r, device="cuda")
        B.rn18op_layernorm_fwd(self.prec, self.x, self.gamma, self.beta, y, self.mean, self.rstd, r, d, self.ldx, d,
                               EPS)
        return y

    def backward(self, dy):
        """The gradient of the forward pass's input, in place of dy unless its
        rows have to be copied."""
        r, d = dy.shape
        if dy.shape != self.x.shape or dy.dtype != self.x.dtype:
            raise ValueError("a gradient of another shape or type than the forward pass's input")
        dy, ld = _rows(dy)
        ws = _workspace(B.rn18op_layernorm_bwd_workspace(self.prec, r, d))
        B.rn18op_layernorm_bwd(self.prec, dy, self.x, self.gamma, self.mean, self.rstd, dy, self.dgamma, self.dbeta, r,
                               d, ld, self.ldx, ld, ws)
        return dy


class Dropout:
    """Dropout of rows whose mask is never stored: rate, seed and the number of
    steps taken, which is held on the device so that a captured step counts on."""

    def __init__(self, p, seed):
        self.p, self.seed = p, seed
        self.steps = torch.zeros(1, dtype=torch.int64, device="cuda")

    def apply(self, x, layer):
        """The rows of x dropped; the same call gives the gradient's."""
        if self.p == 0:
            return x
        x, ld = _rows(x)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        B.rn18op_dropout(_prec(x), x, None, y, *x.shape, ld, 0, x.shape[1], self.p, self.seed, layer << 48, self.steps)
        return y


class RmsNorm:
    """Root-mean-square norm over the last axis of [rows][width], with the
    residual's addition and the branch's dropout in front of it."""

    def __init__(self, width, layer, dropout):
        self.gamma = torch.ones(width, device="cuda")
        self.dgamma = torch.empty_like(self.gamma)
        self.layer, self.dropout = layer, dropout

    def _random(self, p):
        return dict(p=p, seed=self.dropout.seed, step=self.layer << 48, step_add=self.dropout.steps)

    def forward(self, x, res=None, train=True):
        """(h, y): the stream behind the addition, and its norm."""
        r, d = x.shape
        if d != len(self.gamma):
            raise ValueError("rows of %d elements for a norm of %d" % (d, len(self.gamma)))
        if res is not None and (res.shape != x.shape or res.dtype != x.dtype):
            raise ValueError("a residual of another shape or type than the branch")
        x, ldx = _rows(x)
        self.p = self.dropout.p if train and res is not None else 0.0
        h, ldres = (x, 0) if res is None else (torch.empty((r, d), dtype=x.dtype, device=x.device), d)
        if res is not None:
            res, ldres = _rows(res)
        y = torch.empty((r, d), dtype=x.dtype, device=x.device)
        self.rstd = torch.empty(r, device="cuda")
        ldh = ldx if res is None else d
        B.rn18op_rmsnorm_fwd(_prec(x), x, res, self.gamma, None if res is None else h, y, self.rstd, r, d, ldx, ldres,
                             ldh, d, EPS, **self._random(self.p))
        self.h, self.ldh = h, ldh
        return h, y

    def backward(self, dy, dr=None):
        """(gradient of the residual, gradient of the branch) from y's gradient
        and what else the stream's receives."""
        for g in (dy, dr):
            if g is not None and (g.shape != self.h.shape or g.dtype != self.h.dtype):
                raise ValueError("a gradient of another shape or type than the forward pass's input")
        r, d = dy.shape
        dy, lddy = _rows(dy)
        dr, lddr = _rows(dr) if dr is not None else (None, 0)
        ws = _workspace(B.rn18op_rmsnorm_bwd_workspace(_prec(dy), r, d))
        dh = torch.empty((r, d), dtype=dy.dtype, device=dy.device)
        dx = torch.empty_like(dh) if self.p > 0 else None
        B.rn18op_rmsnorm_bwd(_prec(dy), dy, dr, self.h, self.gamma, self.rstd, dh, dx, self.dgamma, r, d, lddy, lddr,
                             self.ldh, d, d, ws=ws, **self._random(self.p))
        return dh, dh if dx is None else dx


class Mixer:
    """Linear attention over the tokens of each sequence: one product for the
    queries, keys and values, which stay in its output's rows, and one behind."""

    def __init__(self, width, heads, generator):
        if width % heads:
            raise ValueError("a width of %d for %d heads" % (width, heads))
        self.heads, self.width, self.dim = heads, width, width // heads
        self.wqkv = torch.randn((width, 3 * width), device="cuda", generator=generator) * width ** -0.5
        self.wo = torch.randn((width, width), device="cuda", generator=generator) * width ** -0.5
        # each head looks back twice as far as the one before it
        self.log_decay = torch.log1p(-torch.exp2(-1.0 - torch.arange(heads, device="cuda", dtype=torch.float32)))

    def _parts(self, qkv):
        return [qkv[:, i * self.width:(i + 1) * self.width] for i in range(3)]

    def forward(self, y, n):
        """The branch of the rows y: n sequences one after the other."""
        if len(y) % n:
            raise ValueError("%d rows of %d sequences" % (len(y), n))
        self.y, self.sizes = y, (n, len(y) // n, self.heads, self.heads, self.dim, self.dim)
        self.qkv = y @ self.wqkv.to(y.dtype)
        self.o = torch.empty((len(y), self.width), dtype=y.dtype, device=y.device)
        ld, p = self.qkv.stride(0), _prec(y)
        ws = _workspace(B.rn18op_linattn_fwd_workspace(p, *self.sizes))
        B.rn18op_linattn_fwd(p, *self._parts(self.qkv), self.log_decay, None, None, self.o, None, *self.sizes, ld, ld, ld,
                             self.width, self.dim ** -0.5, ws)
        return self.o @ self.wo.to(y.dtype)

    def backward(self, dx):
        """The gradient of y; those of the products stay in dwqkv and dwo."""
        self.dwo = (self.o.t() @ dx).float()
        do = dx @ self.wo.to(dx.dtype).t()
        dqkv, p, ld = torch.empty_like(self.qkv), _prec(dx), self.qkv.stride(0)
        ws = _workspace(B.rn18op_linattn_bwd_workspace(p, *self.sizes))
        B.rn18op_linattn_bwd(p, *self._parts(self.qkv), do, self.log_decay, None, None, None, *self._parts(dqkv), None,
                             *self.sizes, ld, ld, ld, do.stride(0), ld, ld, ld, self.dim ** -0.5, ws)
        self.dwqkv = (self.y.t() @ dqkv).float()
        return dqkv @ self.wqkv.to(dx.dtype).t()

    def step(self, y, state):
        """The branch of one token of each sequence, whose state goes on in place."""
        qkv = y @ self.wqkv.to(y.dtype)
        o = torch.empty_like(y)
        ld, h, d = qkv.stride(0), self.heads, self.dim
        B.rn18op_linattn_step(_prec(y), *self._parts(qkv), self.log_decay, state, o, state, len(y), h, h, d, d, ld, ld,
                              ld, o.stride(0), d ** -0.5)
        return o @ self.wo.to(y.dtype)

    def empty_state(self, n):
        return torch.zeros((n, self.heads, self.dim, self.dim), device="cuda")


class TokenStudent:
    """Patches -> product -> layer norm -> [residual blocks] -> ReLU -> mean over
    the patches -> layer norm -> classifier. A block adds the dropped output of a
    mixer of the normed tokens to the stream; the addition, the dropout and the
    next block's norm are one call. The tokens are held in `dtype`, the pooled
    features, logits and parameters in fp32."""

    def __init__(self, classes, width=512, patch=16, dtype=torch.bfloat16, seed=0, blocks=0, heads=8, dropout=0.0):
        if blocks < 0 or heads < 1:
            raise ValueError("%d residual blocks of %d heads" % (blocks, heads))
        if dropout and not blocks:
            raise ValueError("dropout without residual blocks, whose branches it drops")
        g = torch.Generator(device="cuda").manual_seed(seed)
        fan = 3 * patch * patch
        self.patch, self.dtype = patch, dtype
        self.embed = torch.randn((fan, width), device="cuda", generator=g) * fan ** -0.5
        self.head = torch.randn((width, classes), device="cuda", generator=g) * width ** -0.5
        self.bias = torch.zeros(classes, device="cuda")
        self.tokens, self.pooled = LayerNorm(width), LayerNorm(width)
        self.dropout = Dropout(dropout, seed)
        self.mixers = [Mixer(width, heads, g) for _ in range(blocks)]
        self.norms = [RmsNorm(width, i + 1, self.dropout) for i in range(blocks + 1)] if blocks else []
        self.momentum = [torch.zeros_like(p) for p in self.parameters()]

    def parameters(self):
        return [self.embed, self.tokens.gamma, self.tokens.beta, self.pooled.gamma, self.pooled.beta, self.head,
                self.bias] + [m.wqkv for m in self.mixers] + [m.wo for m in self.mixers] + \
            [n.gamma for n in self.norms]

    def patches(self, images):
        n, c, h, w = images.shape
        p = self.patch
        x = images[:, :, :h // p * p, :w // p * p].reshape(n, c, h // p, p, w // p, p)
        return x.permute(0, 2, 4, 1, 3, 5).reshape(-1, c * p * p).to(self.dtype)

    def _blocks(self, a, n, train):
        """The residual blocks on the rows a of n sequences; what the last norm gives."""
        if not self.mixers:
            return a
        h, y = self.norms[0].forward(self.dropout.apply(a, 0) if train else a, None, train)
        for mixer, norm in zip(self.mixers, self.norms[1:]):
            h, y = norm.forward(mixer.forward(y, n), h, train)
        return y

    def _blocks_backward(self, dy):
        if not self.mixers:
            return dy
        dh = None
        for mixer, norm in zip(self.mixers[::-1], self.norms[:0:-1]):
            dh, dx = norm.backward(dy, dh)
            dy = mixer.backward(dx)
        return self.dropout.apply(self.norms[0].backward(dy, dh)[0], 0)

    def gradients(self, images, labels, vals, idx, temperature, alpha):
        """(loss, gradients in the order of parameters()) of one batch."""
        n, (width, classes) = len(images), self.head.shape
        x = self.patches(images)
        a = self._blocks(self.tokens.forward(x @ self.embed.to(self.dtype)), n, True)
        t = len(x) // n
        f = self.pooled.forward(a.relu().view(n, t, width).float().mean(dim=1))
        z = torch.addmm(self.bias, f, self.head)
        k = idx.shape[1]
        row_loss, loss = torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
        need = B.rn18op_distill_loss_workspace(B.RN18_FP32, n, classes, k)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        B.rn18op_distill_loss(B.RN18_FP32, z, vals, idx, labels, None, z, row_loss, loss, n, classes, z.stride(0),
                              z.stride(0), k, temperature, alpha, 1.0 / n, ws)      # z holds its gradient now
        df = self.pooled.backward(z @ self.head.t())
        da = (df / t)[:, None, :].expand(n, t, width).reshape(n * t, width).to(self.dtype) * (a > 0)
        dh = self.tokens.backward(self._blocks_backward(da))
        return loss, [(x.t() @ dh).float(), self.tokens.dgamma, self.tokens.dbeta, self.pooled.dgamma,
                      self.pooled.dbeta, f.t() @ z, z.sum(dim=0)] + [m.dwqkv for m in self.mixers] + \
            [m.dwo for m in self.mixers] + [m.dgamma for m in self.norms]

    def train_step(self, images, labels, vals, idx, temperature, alpha, lr, mu=0.9):
        loss, grads = self.gradients(images, labels, vals, idx, temperature, alpha)
        for p, v, g in zip(self.parameters(), self.momentum, grads):
            v.mul_(mu).add_(g)
            p.sub_(v, alpha=lr)
        self.dropout.steps.add_(1)
        return loss

    def logits(self, images):
        """Evaluation, without dropout."""
        n, width = len(images), self.head.shape[0]
        x = self.patches(images)
        a = self._blocks(self.tokens.forward(x @ self.embed.to(self.dtype)), n, False)
        f = self.pooled.forward(a.relu().view(n, len(x) // n, width).float().mean(dim=1))
        return torch.addmm(self.bias, f, self.head)

    def logits_by_patch(self, images):
        """The same as the patches come in, one of each image at a time."""
        n, width = len(images), self.head.shape[0]
        x = self.patches(images).view(n, -1, self.embed.shape[0])
        states = [m.empty_state(n) for m in self.mixers]
        total = torch.zeros((n, width), device="cuda")
        for t in range(x.shape[1]):
            y = self.tokens.forward(x[:, t] @ self.embed.to(self.dtype))
            if self.mixers:
                h, y = self.norms[0].forward(y, None, False)
                for mixer, norm, state in zip(self.mixers, self.norms[1:], states):
                    h, y = norm.forward(mixer.step(y, state), h, False)
            total += y.relu()
        return torch.addmm(self.bias, self.pooled.forward(total / x.shape[1]), self.head)


def run(student="tokens", arch="imagenet", classes=1000, batch=64, size=128, steps=20, k=10, temperature=4.0,
        alpha=0.9, lr=0.005, prec="bf16", batches=4, log=None, blocks=0, heads=8, dropout=0.0):
    """Trains a student on a few synthetic batches against a network with
    random weights, whose targets are taken once; returns the losses."""
    if student != "tokens" and (blocks or dropout):
        raise ValueError("residual blocks and their dropout are the token student's")
    teacher = B.Worker(arch, classes, prec)
    state = torch.zeros(teacher.n_state, device="cuda")
    B.rn18_destroy(B.rn18_init(teacher.cfg, 1, state))
    data = []
    for i in range(batches):
        x = torch.from_numpy(inputs.images(i, batch, size, size)).cuda()
        y = torch.from_numpy(inputs.labels(i, batch, classes)).cuda()
        data.append((x, y) + teacher_targets(teacher, state, x, k))
    if student == "tokens":
        net = TokenStudent(classes, blocks=blocks, heads=heads, dropout=dropout)
        step = lambda x, y, v, i: net.train_step(x, y, v, i, temperature, alpha, lr)
    else:
        worker = B.Worker(arch, classes, prec)
        params = torch.zeros(worker.n_state, device="cuda")
        B.rn18_destroy(B.rn18_init(worker.cfg, 2, params))
        loss = torch.zeros(1, device="cuda")

        def step(x, y, v, i):
            worker.train_step_distill(params, x, y, v, i, temperature, alpha, lr, loss)
            return loss.clone()
    losses = []
    for s in range(steps):
        losses.append(step(*data[s % batches]))
        if log and s % 10 == 0:
            log("step %d  loss %.4f" % (s, losses[-1].item()))
    if teacher.sync_status() != B.RN18_OK or (student != "tokens" and worker.sync_status() != B.RN18_OK):
        raise RuntimeError(B.rn18_last_error())
    return [float(v.item()) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--student", choices=["tokens", "resnet"], default="tokens")
    ap.add_argument("--arch", choices=["tiny", "cifar", "imagenet"], default="imagenet")
    ap.add_argument("--prec", choices=["fp32", "bf16", "fp16"], default="bf16")
    for name, value in (("classes", 1000), ("batch", 64), ("size", 128), ("steps", 50), ("k", 10), ("batches", 4),
                        ("blocks", 0), ("heads", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    for name, value in (("temperature", 4.0), ("alpha", 0.9), ("lr", 0.005), ("dropout", 0.0)):
        ap.add_argument("--" + name, type=float, default=value)
    run(**vars(ap.parse_args()), log=print)
