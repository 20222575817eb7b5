"""The policy with a layer of experts: its gradients as a whole against float64, and training."""
import torch
import pytest

from paper_2609_09821_amd import binding as im
from paper_2609_09821_amd import experts

pytestmark = pytest.mark.gpu


def _restored(c):
    t = torch.zeros(c.shape, device="cuda")
    im.checkpoint_load(c, t)
    return t.double()


@pytest.mark.parametrize("n,E,dims", [(1, 3, (226, 64, 28)), (500, 5, (361, 96, 69)), (1300, 16, (70, 33, 9))])
def test_gradients_of_the_whole(n, E, dims):
    """Each stage against float64 from the values that it was given, so that every difference
    is that stage's own rounding: 2^-8 of a bf16 result (one rounding of it, and fp32 sums
    far below), 1e-5 of the magnitudes summed for float32 ones."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    p = experts.ExpertPolicy(E, *dims, seed=n)
    b = experts.Batch(p, n)
    b.x.copy_(torch.randn(n, dims[0], device="cuda", generator=g))
    e = torch.randint(-1, E, (n,), device="cuda", dtype=torch.int32, generator=g)
    mean = experts.forward(p, b, e, train=True)
    b.dmean.copy_(torch.randn(n, dims[2], device="cuda", generator=g))
    dgamma, dbeta, dw1, dw2, db1, db2 = experts.backward(p, b)
    ku, kh, kx = _restored(b.keep_u), _restored(b.keep_h), _restored(b.keep_x)
    own = [torch.nonzero(e == k).flatten() for k in range(E)]
    tiny = 1e-12

    def close(got, want, size, rel):
        assert bool(((got.double() - want).abs() <= rel * size + tiny).all())

    xd = b.x.double()
    var, mu = torch.var_mean(xd, 1, unbiased=False, keepdim=True)
    u = (xd - mu) * (var + 1e-5) ** -0.5
    close(b.u, u, u.abs() + 1e-3, 2.0 ** -8)
    seen = torch.zeros(n, dtype=torch.bool, device="cuda")
    for k, r in enumerate(own):
        seen[r] = True
        ud, hd, dm, dh = b.u[r].double(), b.h[r].double(), b.dmean[r].double(), b.dh[r].double()
        w1, w2 = p.w16[0][k].double(), p.w16[1][k].double()
        h = (ud @ w1.t() + p.b[0][k].double()).clamp(min=0)
        close(b.h[r], h, h + 1e-5 * (ud.abs() @ w1.abs().t()) / 2.0 ** -8, 2.0 ** -8)
        close(mean[r], hd @ w2.t() + p.b[1][k].double(), hd.abs() @ w2.abs().t() + 1.0, 1e-5)
        want = (dm @ w2) * (kh[r] > 0)
        close(b.dh[r], want, want.abs() + 1e-5 * (dm.abs() @ w2.abs()) / 2.0 ** -8, 2.0 ** -8)
        close(dw2[k], dm.t() @ kh[r], dm.abs().t() @ kh[r].abs(), 1e-5)
        close(db2[k], dm.sum(0), dm.abs().sum(0), 1e-5)
        close(dw1[k], dh.t() @ ku[r], dh.abs().t() @ ku[r].abs(), 1e-5)
        close(db1[k], dh.sum(0), dh.abs().sum(0), 1e-5)
        want = dh @ w1
        close(b.du[r], want, want.abs() + 1e-5 * (dh.abs() @ w1.abs()) / 2.0 ** -8, 2.0 ** -8)
    assert not mean[~seen].any() and not b.dh[~seen].any() and not b.du[~seen].any()
    hx = (kx - b.row_mean.double()[:, None]) * b.row_rstd.double()[:, None]
    du = b.du.double()
    close(dgamma, (du * hx).sum(0), (du * hx).abs().sum(0), 1e-5)
    close(dbeta, du.sum(0), du.abs().sum(0), 1e-5)


def test_imitation_learns():
    """The loss of an untrained network falls by more than half within 40 steps on moving envs."""
    said = []
    losses = experts.imitate(envs=512, steps=40, log=said.append)
    assert len(losses) == 40 and all(l == l for l in losses)
    assert sum(losses[-5:]) / 5 < 0.5 * losses[0], losses
    assert said


def test_one_env_is_served():
    """A single row, grouped, normed and multiplied as it is served, equals itself in a batch."""
    p = experts.ExpertPolicy(4, 361, 128, 69, seed=2)
    many, one = experts.Batch(p, 40), experts.Batch(p, 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    many.x.copy_(torch.randn(40, 361, device="cuda", generator=g))
    e = torch.randint(0, 4, (40,), device="cuda", dtype=torch.int32, generator=g)
    all_ = experts.forward(p, many, e).clone()
    one.x.copy_(many.x[17:18])
    alone = experts.forward(p, one, e[17:18].contiguous())
    assert torch.equal(alone[0], all_[17])
