"""The distillation example: targets of a teacher, the token student's
gradients against automatic differentiation in 64 bits, and both students
learning."""
import numpy as np
import pytest

from oracle import rows
from paper_2509_26092_amd import binding as B
from paper_2509_26092_amd import inputs

pytestmark = pytest.mark.gpu


def test_teacher_targets_are_its_largest_eval_logits():
    import torch
    from paper_2509_26092_amd import distill
    w = B.Worker("cifar", 100, "fp32")
    state = torch.zeros(w.n_state, device="cuda")
    B.rn18_destroy(B.rn18_init(w.cfg, 3, state))
    x = torch.from_numpy(inputs.images(1, 6, 32, 32)).cuda()
    vals, idx = distill.teacher_targets(w, state, x, 7)
    z = torch.empty((6, 100), device="cuda")
    w.eval_logits(state, x, z)
    v, i = rows.topk(z.cpu().numpy(), 7)
    assert np.array_equal(idx.cpu().numpy(), i) and np.array_equal(vals.cpu().numpy(), v)


def test_token_student_gradients():
    """fp32 against float64: sums of up to 10 x 768 products and two layer
    norms, a few hundred roundings of 2^-24 each; 1e-4 of a tensor's norm."""
    import torch
    from paper_2509_26092_amd import distill
    n, classes, k, temp, alpha = 10, 50, 6, 2.0, 0.6
    s = distill.TokenStudent(classes, width=96, dtype=torch.float32, seed=4)
    s.tokens.gamma.normal_(1.0, 0.2)
    s.tokens.beta.normal_(0.0, 0.2)
    s.pooled.gamma.normal_(1.0, 0.2)
    rng = np.random.default_rng(2)
    x = torch.from_numpy(inputs.images(2, n, 50, 36)).cuda()      # 3 x 2 patches, the rest cut off
    y = torch.from_numpy(inputs.labels(2, n, classes)).cuda()
    idx = torch.from_numpy(np.stack([rng.permutation(classes)[:k] for _ in range(n)]).astype(np.int32)).cuda()
    vals = torch.from_numpy((rng.standard_normal((n, k)) * 2).astype(np.float32)).cuda()
    loss, grads = s.gradients(x, y, vals, idx, temp, alpha)

    p = [t.detach().cpu().double().requires_grad_() for t in s.parameters()]
    F = torch.nn.functional
    h = F.layer_norm(s.patches(x).cpu().double() @ p[0], (96,), p[1], p[2], distill.EPS).relu()
    f = F.layer_norm(h.view(n, -1, 96).mean(1), (96,), p[3], p[4], distill.EPS)
    z = f @ p[5] + p[6]
    q = torch.softmax(vals.cpu().double() / temp, 1)
    lp = torch.log_softmax(z / temp, 1).gather(1, idx.cpu().long())
    want = (alpha * temp ** 2 * (q * (q.log() - lp)).sum(1)).mean() + (1 - alpha) * F.cross_entropy(z, y.cpu().long())
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()
    for i, (g, t) in enumerate(zip(grads, p)):
        assert (g.cpu().double() - t.grad).norm() <= 1e-4 * t.grad.norm(), i


@pytest.mark.parametrize("student,arch,classes,size,prec", [("tokens", "cifar", 100, 32, "fp32"),
                                                            ("tokens", "imagenet", 1000, 64, "bf16"),
                                                            ("resnet", "cifar", 100, 32, "bf16")])
def test_students_learn(student, arch, classes, size, prec):
    from paper_2509_26092_amd import distill
    losses = distill.run(student, arch, classes, 16, size, 24, prec=prec, batches=2)
    assert np.isfinite(losses).all()
    assert np.mean(losses[-4:]) < 0.8 * np.mean(losses[:4])
