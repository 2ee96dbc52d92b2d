"""The token student with residual blocks: dropout, RMS norm and linear
attention together, as training, evaluation and serving use them."""
import numpy as np
import pytest

from oracle import rows
from paper_2509_26092_amd import binding as B, inputs

pytestmark = pytest.mark.gpu


def batch(n, classes, k, size=(50, 36)):
    import torch
    rng = np.random.default_rng(2)
    x = torch.from_numpy(inputs.images(2, n, *size)).cuda()
    y = torch.from_numpy(inputs.labels(2, n, classes)).cuda()
    idx = torch.from_numpy(np.stack([rng.permutation(classes)[:k] for _ in range(n)]).astype(np.int32)).cuda()
    vals = torch.from_numpy((rng.standard_normal((n, k)) * 2).astype(np.float32)).cuda()
    return x, y, vals, idx


def attention(q, k, v, log_decay):
    """[n][t][heads][d] in 64 bits, the quadratic form."""
    import torch
    t, d = q.shape[1], q.shape[3]
    i = torch.arange(t)
    lag = (i[:, None] - i[None, :]).clamp(min=0)
    w = torch.exp(log_decay[:, None, None] * lag) * (i[:, None] >= i[None, :])
    p = (q.transpose(1, 2) @ k.transpose(1, 2).transpose(2, 3)) * w
    return (p @ v.transpose(1, 2)).transpose(1, 2) * d ** -0.5


@pytest.mark.parametrize("p", [0.0, 0.2])
def test_gradients_of_the_blocks(p):
    """fp32 against automatic differentiation in 64 bits with the generator's
    masks: sums of up to 10 x 768 products through two blocks, a few hundred
    roundings of 2^-24 each; 1e-4 of a tensor's norm."""
    import torch
    from paper_2509_26092_amd import distill
    n, classes, k, temp, alpha, width, heads, blocks = 10, 50, 6, 2.0, 0.6, 96, 4, 2
    s = distill.TokenStudent(classes, width=width, patch=8, dtype=torch.float32, seed=4, blocks=blocks, heads=heads,
                             dropout=p)
    for g in [s.tokens.gamma, s.pooled.gamma] + [m.gamma for m in s.norms]:
        g.normal_(1.0, 0.2)
    s.tokens.beta.normal_(0.0, 0.2)
    s.dropout.steps.fill_(5)
    x, y, vals, idx = batch(n, classes, k)                          # 6 x 4 patches
    loss, grads = s.gradients(x, y, vals, idx, temp, alpha)

    q = [t.detach().cpu().double().requires_grad_() for t in s.parameters()]
    embed, tg, tb, pg, pb, head, bias = q[:7]
    wqkv, wo, gammas = q[7:7 + blocks], q[7 + blocks:7 + 2 * blocks], q[7 + 2 * blocks:]
    F = torch.nn.functional
    R, t = n * 24, 24
    mask = lambda layer: torch.from_numpy(rows.dropout_factor(4, (layer << 48) + 5, R, width, p))
    rms = lambda h, g: h / torch.sqrt((h * h).mean(1, keepdim=True) + distill.EPS) * g
    h = F.layer_norm(s.patches(x).cpu().double() @ embed, (width,), tg, tb, distill.EPS) * mask(0)
    a = rms(h, gammas[0])
    for i in range(blocks):
        qkv = (a @ wqkv[i]).view(n, t, 3, heads, width // heads)
        o = attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], s.mixers[i].log_decay.cpu().double())
        h = h + mask(i + 2) * (o.reshape(R, width) @ wo[i])
        a = rms(h, gammas[i + 1])
    f = F.layer_norm(a.relu().view(n, t, width).mean(1), (width,), pg, pb, distill.EPS)
    z = f @ head + bias
    soft = torch.softmax(vals.cpu().double() / temp, 1)
    lp = torch.log_softmax(z / temp, 1).gather(1, idx.cpu().long())
    want = (alpha * temp ** 2 * (soft * (soft.log() - lp)).sum(1)).mean() + \
        (1 - alpha) * F.cross_entropy(z, y.cpu().long())
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()
    for i, (g, w) in enumerate(zip(grads, q)):
        assert (g.cpu().double() - w.grad).norm() <= 1e-4 * w.grad.norm(), i


@pytest.mark.parametrize("prec,tol", [("float32", 2e-4), ("bfloat16", 0.1)])
def test_patch_by_patch_gives_the_whole_images_logits(prec, tol):
    """Single tokens with carried states against whole sequences. fp32: a few
    hundred roundings of 2^-24; bf16: some twenty stored tensors in a row, 2^-8
    each, in quadrature 2^-8 sqrt(20) = 0.02 and five times that."""
    import torch
    from paper_2509_26092_amd import distill
    s = distill.TokenStudent(20, width=128, patch=8, dtype=getattr(torch, prec), seed=1, blocks=2, heads=2,
                             dropout=0.5)
    x = batch(5, 20, 3, (64, 64))[0]
    a, b = s.logits(x), s.logits_by_patch(x)
    assert torch.equal(a, s.logits(x))                               # no dropout
    assert (a - b).norm() <= tol * a.norm()


def test_a_captured_step_counts_on():
    """Replays of a captured training step against eager steps of a student of
    the same seed: other masks each step, the same losses and parameters."""
    import torch
    from paper_2509_26092_amd import distill
    make = lambda: distill.TokenStudent(20, width=128, patch=8, dtype=torch.float32, seed=3, blocks=1, heads=2,
                                        dropout=0.3)
    data = batch(4, 20, 3, (32, 32))
    step = lambda s: s.train_step(*data, 2.0, 0.6, 0.02)
    a, b = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [step(a).clone(), step(b).clone()]                    # (workspaces and libraries set up)
    torch.cuda.synchronize()
    assert torch.equal(*want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss = step(b)
    losses = []
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got, ref = loss.clone(), step(a)
        torch.cuda.synchronize()
        assert abs(got.item() - ref.item()) <= 1e-5 * abs(ref.item())
        losses.append(got.item())
    assert b.dropout.steps.item() == 5 and len(set(losses)) == 4
    for p, q in zip(a.parameters(), b.parameters()):
        assert (p - q).norm() <= 1e-5 * p.norm()


def test_the_command_runs_with_blocks():
    from paper_2509_26092_amd import distill
    losses = distill.run("tokens", "cifar", 100, 8, 32, 4, prec="bf16", batches=2, blocks=2, heads=4, dropout=0.1)
    assert len(losses) == 4 and np.isfinite(losses).all()


def test_a_captured_step_has_scratch_of_its_own():
    """A captured step's workspaces are not those of eager steps, which a larger
    batch would replace, so that replays would write to memory given back."""
    import torch
    from paper_2509_26092_amd import distill
    make = lambda: distill.TokenStudent(20, width=128, patch=8, dtype=torch.float32, seed=4, blocks=1, heads=1)
    data, larger = batch(2, 20, 3, (160, 160)), batch(3, 20, 3, (192, 192))
    step = lambda s: s.train_step(*data, 2.0, 0.6, 0.02)
    a, b = make(), make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a), step(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss = step(b)
    sizes = [B.rn18op_linattn_bwd_workspace(0, 2, 400, 1, 1, 128, 128), B.rn18op_rmsnorm_bwd_workspace(0, 800, 128)]
    assert all(sizes)
    with torch.cuda.stream(side):
        b.gradients(*larger, 2.0, 0.6)
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        got, ref = loss.clone(), step(a)
        torch.cuda.synchronize()
        assert abs(got.item() - ref.item()) <= 1e-5 * abs(ref.item())
        assert all((t == 7).all() for t in others)


def test_the_layers_refuse_other_shapes_and_types():
    import torch
    from paper_2509_26092_amd import distill
    d = distill.Dropout(0.0, 1)
    norm, mixer = distill.RmsNorm(16, 1, d), distill.Mixer(16, 2, torch.Generator(device="cuda").manual_seed(1))
    x = torch.ones((6, 16), device="cuda")
    for args in ((x[:, :8],), (x, x[:3]), (x, x.bfloat16())):
        with pytest.raises(ValueError):
            norm.forward(*args)
    norm.forward(x, x)
    for args in ((x[:3],), (x.bfloat16(),), (x, x[:3]), (x, x.bfloat16())):
        with pytest.raises(ValueError):
            norm.backward(*args)
    with pytest.raises(ValueError):
        mixer.forward(x, 4)
