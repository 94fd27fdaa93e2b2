"""Products with 4-bit weights where a row of x holds infinities, or values so large that sums over codes pass the largest float: every entry is what
the definition gives, whichever kernel serves the call and however many rows are in it."""
import pytest
import torch

from test_gpu_q4 import F, FLOATS, apart, dense, ints, packed, rng, weights, wide  # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")
# rows of every kernel: a wave's own (1, 2 rows), staged (to 5 in fp32, to 16), tiles of each size; sums divided over work-groups (8192 and 6000 columns)
SIZES = [(1, 300, 90), (2, 300, 90), (3, 260, 33), (5, 300, 90), (6, 520, 90), (16, 300, 40), (17, 300, 90), (40, 300, 90), (6, 6000, 40), (40, 8192, 70), (20, 6000, 36),
         (200, 256, 900), (300, 130, 1100), (700, 140, 300)]


def by_definition(x, w):
    """sum over c of x[m][c] w[k][c] in 64 bits, each product formed (0 times infinity is NaN)."""
    return torch.stack([(row * w).sum(1) for row in x.double().cpu()]).cuda()


def same(got, want):
    return bool((torch.isnan(got) == torch.isnan(want)).all()) and torch.equal(got.nan_to_num(0, 1e30, -1e30), want.nan_to_num(0, 1e30, -1e30))


@pytest.mark.parametrize("xt", FLOATS, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,c,k", SIZES)
def test_infinite(F, m, c, k, xt):  # noqa: F811
    """Integers and scales that are powers of two, exact in 32 bits; in the first row one infinity, in the last one another, in the second
    to last (of three and more) one of each sign."""
    case = SIZES.index((m, c, k))
    group, zeros = (32, 64, 128)[case % 3], case % 2 == 0
    g = rng(case)
    q, s, z = weights(g, k, c, group, zeros, powers=True)
    h = F.q4_import(packed(q), s, z, group=group, c=c)
    w = dense(q, s, z, group)[0].cpu()
    x = ints(g, -3, 4, m, c).to(xt)
    finite = F.linear_q4(h, x, out_dtype=torch.float32)
    x[0, c - 1] = INF
    x[-1, c // 2] = -INF
    if m > 2:
        x[-2, 1], x[-2, c - 2] = INF, -INF
    rows = sorted({0, m - 1} | ({m - 2} if m > 2 else set()))
    want = finite.double()
    want[rows] = by_definition(x[rows], w)
    assert bool((want[0] == INF).any()) and bool((want[0] == -INF).any()) and bool(torch.isnan(want[rows]).any())
    for a in (x, apart(x, 3, 1)):
        assert same(F.linear_q4(h, a, out_dtype=torch.float32), want.float())
        assert same(F.linear_q4(h, a), want.to(xt))
        leaky = F.linear_q4(h, a, leaky=0.5, out_dtype=torch.float32)
        assert same(leaky, torch.where(want > 0, want, 0.5 * want).float())
        relu = F.linear_q4(h, a, relu=True, out_dtype=torch.float32)
        known = ~torch.isnan(want)
        assert torch.equal(relu[known], want.clamp(min=0).float()[known])


@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,c,k", SIZES)
def test_the_largest(F, m, c, k, xt):  # noqa: F811
    """x of up to 3 * 2^126, scales 2^-22 to 2^-19: the sums of a group pass the largest float, results are multiples of 2^104 below c * 45 * 2^107 and
    exact."""
    case = SIZES.index((m, c, k))
    group = (64, 128, 32)[case % 3]
    g = rng(case)
    q, s, z = weights(g, k, c, group, True, powers=True)
    s = s * 2.0 ** -20
    h = F.q4_import(packed(q), s, z, group=group, c=c)
    x = ints(g, -3, 4, m, c).float() * 2.0 ** 126
    x[m // 2] *= 2.0 ** -126                           # a row of ordinary values among them
    x = x.to(xt)
    want = x.double() @ dense(q, s, z, group)[0].t()
    bias = ints(g, -5, 6, k).float() * 2.0 ** 110
    assert float(want.abs().max()) < 2.0 ** 126
    assert torch.equal(F.linear_q4(h, x, out_dtype=torch.float32).double(), want)
    keep = [i for i in range(m) if i != m // 2]
    assert torch.equal(F.linear_q4(h, x, bias=bias, relu=True)[keep], (want + bias.double()).clamp(min=0).to(xt)[keep])


@pytest.mark.parametrize("rows", [False, True], ids=["groups", "rows"])
@pytest.mark.parametrize("m", [1, 3, 16, 40, 300])
def test_eight_bits_with_scales_at_both_ends(F, m, rows):  # noqa: F811
    """Scales of x of 2^124 and of the weights of 2^-122, and a scale that is infinite: the definition's values."""
    g = rng(m)
    c, k, group = 300, 90, 64
    q, s, z = weights(g, k, c, group, True, powers=True)
    s = s * 2.0 ** -122
    h = F.q4_import(packed(q), s, z, group=group, c=c)
    w = dense(q, s, z, group)[0]
    x = ints(g, -3, 4, m, c).to(torch.int8)
    xs = torch.full((m,) if rows else (m, (c + group - 1) // group), 2.0 ** 124, device="cuda")
    x64 = x.double() * (xs.double()[:, None] if rows else wide(xs, group, c))
    assert torch.equal(F.linear_q4(h, x, x_scale=xs).double(), x64 @ w.t())
    xs.view(m, -1)[0, 0] = INF
    x64 = x.double() * (xs.double()[:, None] if rows else wide(xs, group, c))
    want = x64 @ w.t()
    want[0] = by_definition(x64[:1], w.cpu())
    assert same(F.linear_q4(h, x, x_scale=xs), want.float())


@pytest.mark.parametrize("xt", FLOATS + [torch.int8], ids=["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("m", [1, 5, 16, 40, 300])
def test_nan_through_the_activation(F, m, xt):  # noqa: F811
    """What is NaN before a ReLU or LeakyReLU is NaN behind it, and nothing else is: of x, of its scales, of the bias."""
    g = rng(m)
    c, k = 300, 90
    q, s, z = weights(g, k, c, 64, True, powers=True)
    h = F.q4_import(packed(q), s, z, group=64, c=c)
    x = ints(g, -3, 4, m, c).to(xt)
    xs = torch.ones(m, device="cuda") if xt == torch.int8 else None
    bias = ints(g, -5, 6, k).float()
    bias[7], bias[8], bias[9] = float("nan"), INF, -INF
    want = x.double() @ dense(q, s, z, 64)[0].t() + bias.double()
    if xs is None:
        x[-1, 3] = float("nan")
    else:
        xs[-1] = float("nan")
    want[-1] = float("nan")
    for act, y in ((dict(relu=True), want.clamp(min=0)), (dict(leaky=0.5), torch.where(want > 0, want, want * 0.5)), ({}, want)):
        for yt in FLOATS:
            got = F.linear_q4(h, x, bias=bias, x_scale=xs, out_dtype=yt, **act)
            assert same(got, y.to(yt)) and not bool(torch.signbit(got[got == 0]).any())


@pytest.mark.parametrize("m", [1, 5, 8, 16, 40, 300])
def test_the_smallest(F, m):  # noqa: F811
    """16-bit x is exact down to its smallest number.  fp32 x enters with what bfloat16 holds of it, steps of 2^-133 and up: a term is off by less than that times
    the weight's magnitude, scale (code + zero), whatever else rounds (n roundings of the sum, as for ordinary values)."""
    g = rng(m)
    c, k = 300, 90
    q, s, z = weights(g, k, c, 64, True, powers=True)
    s = s * 2.0 ** 20
    h = F.q4_import(packed(q), s, z, group=64, c=c)
    w, most = dense(q, s, z, 64)
    for xt, e in ((torch.float16, -24), (torch.bfloat16, -126), (torch.bfloat16, -133), (torch.float32, -126), (torch.float32, -133)):
        x = (ints(g, -3, 4, m, c).double() * 2.0 ** e).to(xt)
        assert torch.equal(F.linear_q4(h, x, out_dtype=torch.float32).double(), x.double() @ w.t())
    for e in (-100, -115, -125, -140):
        x = torch.randn(m, c, generator=g, device="cuda") * 2.0 ** e
        want = x.double() @ w.t()
        got = F.linear_q4(h, x).double()
        bound = 2.0 ** -133 * most.sum(1) + 2 * (c + 8) * 2.0 ** -24 * (x.double().abs() @ most.t())
        assert bool(((got - want).abs() <= bound).all())


@pytest.mark.parametrize("xt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("m,c,k", SIZES)
def test_nan_beside_infinities_and_the_largest(F, m, c, k, xt):  # noqa: F811
    """A NaN anywhere in a row of x makes all of its outputs NaN, whatever else the row holds; rows around it are the definition's."""
    case = SIZES.index((m, c, k))
    g = rng(case)
    q, s, z = weights(g, k, c, 64, True, powers=True)
    s = s * 2.0 ** -20
    h = F.q4_import(packed(q), s, z, group=64, c=c)
    w = dense(q, s, z, 64)[0]
    x = (ints(g, -3, 4, m, c).float() * 2.0 ** 126).to(xt)
    want = x.double() @ w.t()
    for row, col in ((0, c - 1), (m // 2, 0), (m - 1, c // 2)):
        x[row, col] = float("nan")
        want[row] = float("nan")
    x[0, 0] = INF
    x[m - 1, 1] = -INF
    for a in (x, apart(x, 3, 1)):
        assert same(F.linear_q4(h, a, out_dtype=torch.float32), want.float())
        assert same(F.linear_q4(h, a, relu=True), want.clamp(min=0).to(xt))
