"""Distillation from a trained network: the teacher's top logits are kept once
a batch, and a student learns from them and the labels.

Two students: the library's own ResNet-18 step (Worker.train_step_distill),
and TokenStudent, a small network of patches with layer norm over channels,
whose forward and backward passes call the row operators (its products, ReLU
and means are torch's, as in a network of the user's).

    python -m paper_2509_26092_amd.distill --student tokens --steps 50
"""
import argparse

import torch

from . import binding as B
from . import inputs

EPS = 1e-5


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


class LayerNorm:
    """Layer norm over the last axis of [rows][width]: parameters, what the
    backward pass needs, and gradients."""

    def __init__(self, width):
        self.gamma, self.beta = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.dgamma, self.dbeta = torch.empty_like(self.gamma), torch.empty_like(self.beta)
        self.ws = None

    def forward(self, x):
        r, d = x.shape
        if d != len(self.gamma):
            raise ValueError("rows of %d elements for a layer norm of %d" % (d, len(self.gamma)))
        self.prec = {torch.float32: B.RN18_FP32, torch.bfloat16: B.RN18_BF16, torch.float16: B.RN18_FP16}[x.dtype]
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
        need = B.rn18op_layernorm_bwd_workspace(self.prec, r, d)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        B.rn18op_layernorm_bwd(self.prec, dy, self.x, self.gamma, self.mean, self.rstd, dy, self.dgamma, self.dbeta, r,
                               d, ld, self.ldx, ld, self.ws)
        return dy


class TokenStudent:
    """Patches -> product -> layer norm -> ReLU -> mean over the patches ->
    layer norm -> classifier. The tokens are held in `dtype`, the pooled
    features, logits and parameters in fp32."""

    def __init__(self, classes, width=512, patch=16, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        fan = 3 * patch * patch
        self.patch, self.dtype = patch, dtype
        self.embed = torch.randn((fan, width), device="cuda", generator=g) * fan ** -0.5
        self.head = torch.randn((width, classes), device="cuda", generator=g) * width ** -0.5
        self.bias = torch.zeros(classes, device="cuda")
        self.tokens, self.pooled = LayerNorm(width), LayerNorm(width)
        self.momentum = [torch.zeros_like(p) for p in self.parameters()]

    def parameters(self):
        return [self.embed, self.tokens.gamma, self.tokens.beta, self.pooled.gamma, self.pooled.beta, self.head,
                self.bias]

    def patches(self, images):
        n, c, h, w = images.shape
        p = self.patch
        x = images[:, :, :h // p * p, :w // p * p].reshape(n, c, h // p, p, w // p, p)
        return x.permute(0, 2, 4, 1, 3, 5).reshape(-1, c * p * p).to(self.dtype)

    def gradients(self, images, labels, vals, idx, temperature, alpha):
        """(loss, gradients in the order of parameters()) of one batch."""
        n, (width, classes) = len(images), self.head.shape
        x = self.patches(images)
        a = self.tokens.forward(x @ self.embed.to(self.dtype))
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
        dh = self.tokens.backward(da)
        return loss, [(x.t() @ dh).float(), self.tokens.dgamma, self.tokens.dbeta, self.pooled.dgamma,
                      self.pooled.dbeta, f.t() @ z, z.sum(dim=0)]

    def train_step(self, images, labels, vals, idx, temperature, alpha, lr, mu=0.9):
        loss, grads = self.gradients(images, labels, vals, idx, temperature, alpha)
        for p, v, g in zip(self.parameters(), self.momentum, grads):
            v.mul_(mu).add_(g)
            p.sub_(v, alpha=lr)
        return loss


def run(student="tokens", arch="imagenet", classes=1000, batch=64, size=128, steps=20, k=10, temperature=4.0,
        alpha=0.9, lr=0.005, prec="bf16", batches=4, log=None):
    """Trains a student on a few synthetic batches against a network with
    random weights, whose targets are taken once; returns the losses."""
    teacher = B.Worker(arch, classes, prec)
    state = torch.zeros(teacher.n_state, device="cuda")
    B.rn18_destroy(B.rn18_init(teacher.cfg, 1, state))
    data = []
    for i in range(batches):
        x = torch.from_numpy(inputs.images(i, batch, size, size)).cuda()
        y = torch.from_numpy(inputs.labels(i, batch, classes)).cuda()
        data.append((x, y) + teacher_targets(teacher, state, x, k))
    if student == "tokens":
        net = TokenStudent(classes)
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
    for name, value in (("classes", 1000), ("batch", 64), ("size", 128), ("steps", 50), ("k", 10), ("batches", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    for name, value in (("temperature", 4.0), ("alpha", 0.9), ("lr", 0.005)):
        ap.add_argument("--" + name, type=float, default=value)
    run(**vars(ap.parse_args()), log=print)
