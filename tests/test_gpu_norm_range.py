"""The root-mean-square norm where squares leave the range of 32 bits: rows of the largest and of the smallest values, which have the definition's
results as ordinary rows do, and rows that hold both."""
import pytest
import torch

from test_gpu_rms_norm import F, FLOATS, apart, randn, rng, slack  # noqa: F401

pytestmark = pytest.mark.gpu
# rows of eight threads to 1024, one vector a thread to sixteen
LENGTHS = [1, 7, 64, 100, 256, 512, 1000, 2048, 4096, 5000, 16384, 30000, 65536]


def definition(h, eps):
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)


@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d", LENGTHS)
def test_both_ends(F, d, xt):  # noqa: F811
    """Rows times powers of two from 2^-120 to 2^120: x / rms(x) does not change, for eps far below (0) and, at the upper end, for an ordinary one.  y is off by
    slack() and by half a step of its type."""
    g = rng(d)
    x = randn(g, 6, d) + 2.0
    exps = torch.tensor([120.0, 90.0, 65.0, -60.0, -90.0, -120.0], device="cuda")
    x = (x.to(xt).float() * torch.exp2(exps)[:, None]).to(xt)
    w = (1 + 0.3 * randn(g, d)).to(xt)
    for eps in (0.0, 1e-5):
        for a in (x, apart(x, 3, 1)):
            y = definition(x.double(), eps) * w.double()
            got = F.rms_norm(a, w, eps)
            # (an fp32 y below the smallest normal number has steps of 2^-149; at eps = 1e-5 rows are x * 316)
            tol = y.abs() * (slack(d) + torch.finfo(xt).eps / 2 * (1 + slack(d))) + 2.0 ** -130
            assert bool(((got.double() - y).abs() <= tol).all())
        for group in (0, 64):
            q, s = F.rms_norm_q8(x, w, eps, group=group)
            step = group or d
            wide = s.double().view(6, -1).repeat_interleave(step, 1)[:, :d]
            rows = slice(0, 6 if eps == 0 else 3)         # (the others' scales are below the normal numbers)
            assert bool(((q.double() * wide - y).abs() <= wide * (0.5 + 127 * 8 * 2.0 ** -24) + y.abs() * slack(d))[rows].all())
            assert int(q[rows].abs().max()) == 127


@pytest.mark.parametrize("d", LENGTHS)
def test_the_residual_s_sum(F, d):  # noqa: F811
    """h = x + r near the largest float, and of the smallest numbers there are, below the normal ones."""
    g = rng(d)
    x, r = randn(g, 4, d).clamp(-3, 3), randn(g, 4, d).clamp(-3, 3)
    x[:2] *= 2.0 ** 124
    r[:2] *= 2.0 ** 124
    x[2:] = torch.round(x[2:] * 8) * 2.0 ** -149
    r[2:] = torch.round(r[2:] * 8) * 2.0 ** -149
    x[2:, 0] = 5 * 2.0 ** -149                            # (no row of zeros)
    r[2:, 0] = 0
    y, h = F.rms_norm(x, None, 0.0, residual=r)
    h64 = (x + r).double()                                # (h is rounded to 32 bits before it is squared)
    assert torch.equal(h, x + r)
    want = definition(h64, 0.0)
    assert bool(((y.double() - want).abs() <= want.abs() * (slack(d) + 2.0 ** -24)).all())


def test_what_stays(F):  # noqa: F811
    """Rows of zeros without eps have no norm; one infinity makes the rest of its row zero; one of the largest values among ordinary ones."""
    x = randn(rng(1), 5, 300)
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 5] = 2.0 ** 120
    x[3] *= 2.0 ** -100
    x[3, 7] = 2.0 ** 100
    y = F.rms_norm(x, None, 0.0)
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isnan(y[1, 5])) and not y[1, :5].any()
    for i in (2, 3, 4):
        want = definition(x[i:i + 1].double(), 0.0)[0]
        assert bool(((y[i].double() - want).abs() <= want.abs() * (slack(300) + 2.0 ** -24) + 2.0 ** -140).all())
    assert not F.rms_norm(x, None, 1e-5)[0].any()
