"""The student block's operators together, as examples/student.py uses them: the gradients of
a whole step against torch's differentiation of the same block in fp64, and a short run
that has to learn."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# From the loss back to the first parameter about 16 tensors are rounded to bf16 one after
# the other (2^-9 of their size as a root mean square: half a step of 8 bits over sqrt 3 is
# below that), independently: 16^(1/2) 2^-9 = 0.8 %, with what each norm and product passes
# on.  Held to 3 % of the norm.
TOL = 3e-2


@pytest.fixture(scope="module")
def student():
    spec = importlib.util.spec_from_file_location("student", os.path.join(ROOT, "examples",
                                                                          "student.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(student, p, ids, teacher, target, weight, tau):
    """The loss of every position by torch, fp64."""
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    B, n = ids.shape
    d = q["E"].shape[1]

    def rms(v, w):
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + student.EPS) * w

    r = q["E"][ids.view(-1).long()]
    x = rms(r, q["n0"]).view(B, n, d)
    for l in range(q["W_self"].shape[0]):
        k = 4 << l
        pos = torch.arange(n, device=ids.device)
        takes = ((pos // k) % 2 == 1).double()[None, :, None]
        back = torch.roll(x, k, dims=1) * takes
        x = x @ q["W_self"][l].T + back @ q["W_nbr"][l].T
    r = r + q["g1"] * rms(x.reshape(B * n, d), q["m1"])
    x = rms(r, q["n1"])
    h = q["W2"].shape[1]
    gu = x @ q["W1"].T
    f = (torch.nn.functional.silu(gu[:, :h]) * gu[:, h:]) @ q["W2"].T
    r = r + q["g2"] * rms(f, q["m2"])
    z = rms(r, q["n2"]) @ q["Wh"].T
    at, t = teacher
    pt = torch.softmax(t.double() / tau, -1)
    lq = torch.log_softmax(z / tau, -1).gather(1, at.long())
    kl = (pt * (pt.log() - lq)).sum(-1) * tau * tau
    ce = torch.nn.functional.cross_entropy(z, target.long(), reduction="none")
    loss = weight.double() * (0.5 * kl + 0.5 * ce)
    grads = torch.autograd.grad(loss.sum(), list(q.values()))
    return loss.detach(), dict(zip(q, grads))


@pytest.mark.parametrize("B,n,V,d,h,L", [(3, 32, 97, 64, 136, 1), (2, 64, 200, 192, 256, 2)])
def test_a_step_is_the_blocks_gradient(student, B, n, V, d, h, L):
    gen = torch.Generator(device="cuda").manual_seed(d)
    table = 2.0 * torch.randn(2, V, V, generator=gen, device="cuda")
    p = student.init(V, d, h, L, seed=3)
    ids, teacher, target = student.batch(table, V, B, n, 12, gen)
    weight = torch.full((B * n,), 1.0 / (B * n), device="cuda")
    loss, g = student.step(p, ids, teacher, target, weight, temperature=2.0)
    rl, rg = reference(student, p, ids, teacher, target, weight, 2.0)
    assert set(g) == set(p)
    assert float((loss.double() - rl).norm() / rl.norm()) < TOL
    for k in p:
        assert g[k].shape == p[k].shape
        err = float((g[k].double() - rg[k]).norm() / rg[k].norm())
        assert err < TOL, (k, err)


def test_a_short_run_learns(student):
    """The label's cross-entropy alone starts at ln V = 4.6; the teacher's own entropy is far
    below it, so the joint loss has to come down clearly within forty steps."""
    losses = student.train(steps=40, say=None)
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0]
