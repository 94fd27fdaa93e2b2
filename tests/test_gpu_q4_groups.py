"""Products with 4-bit weights: every kernel with every group size, in one process, bit for bit on integers."""
import pytest
import torch

from test_gpu_q4 import F, FLOATS, apart, dense, ints, packed, rng, weights, wide  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = FLOATS + [torch.int8]
IDS = ["f32", "f16", "bf16", "i8"]


def check(F, m, c, k, xt, group, zeros, rows, views=("tight",)):
    """x in -1..1, codes and zero points 0..15, scales that are powers of two from 1/4 to 2 (int8 x has scales of 1/2 and 1, by row or by group): sums are multiples of
    1/8 that 32 bits hold."""
    g = rng(m + c + k + group)
    q, s, z = weights(g, k, c, group, zeros, powers=True)
    h = F.q4_import(packed(q), s, z, group=group, c=c)
    x = ints(g, -1, 2, m, c).to(xt)
    xs, x64 = None, x.double()
    if xt == torch.int8:
        xs = torch.exp2(ints(g, -1, 1, m).float()) if rows else torch.exp2(ints(g, -1, 1, m, (c + group - 1) // group).float())
        x64 = x64 * (xs.double()[:, None] if rows else wide(xs, group, c))
    want = x64 @ dense(q, s, z, group)[0].t()
    e = 16 // x.element_size()
    for v in views:
        a = x if v == "tight" else apart(x, (-c) % e + e) if v == "apart" else apart(x, 1, 3)
        assert torch.equal(F.linear_q4(h, a, x_scale=xs, out_dtype=torch.float32).double(), want)


@pytest.mark.parametrize("xt", TYPES, ids=IDS)
@pytest.mark.parametrize("m,c,k", [(16, 4100, 500), (3, 25088, 300), (5, 25088, 300), (16, 9000, 64), (8, 8192, 4000)])
def test_more_than_64_kb_of_rows(F, m, c, k, xt):  # noqa: F811
    """Rows that are staged in up to 144 KB of LDS, in one turn or several, with each group size after the other."""
    for group in (128, 32, 64):
        check(F, m, c, k, xt, group, group != 64, group == 32)
