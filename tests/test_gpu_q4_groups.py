"""Products with 4-bit weights: every kernel with every group size, in one process, bit for bit on integers."""
import pytest
import torch

from test_gpu_q4 import F, FLOATS, apart, dense, ints, packed, rng, weights, wide  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = FLOATS + [torch.int8]
IDS = ["f32", "f16", "bf16", "i8"]


def check(F, m, c, k, xt, group, zeros, rows, views=("tight",), extra=()):
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
    if "no room" in extra:                             # and without scratch, whatever the call would like to have
        y = torch.zeros(m, k, device="cuda")
        st = F._native().linear_q4(h.address, a.data_ptr(), F._DTYPES[xt], a.stride(0), None if xs is None else xs.data_ptr(), 1 if xs is None or rows else xs.shape[1],
                                   m, c, None, 1.0, y.data_ptr(), F.F32, k, None, 0, torch.cuda.current_stream().cuda_stream)
        assert st == 0 and torch.equal(y.double(), want)
    if "room" in extra:                                # the scratch that is asked for is used, and no more of it
        need = F._native().linear_q4_workspace(h.address, F._DTYPES[xt], m)
        assert need > 0
        ws = torch.full((need // 4 + 64,), 7.0, device="cuda")
        F._native().linear_q4(h.address, a.data_ptr(), F._DTYPES[xt], a.stride(0), None if xs is None else xs.data_ptr(), 1 if xs is None or rows else xs.shape[1],
                              m, c, None, 1.0, y.data_ptr(), F.F32, k, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(y.double(), want) and bool((ws[need // 4:] == 7).all()) and not bool((ws[:need // 4].view(-1, (k + 15) // 16 * 16)[:, :k] == 7).all())


@pytest.mark.parametrize("xt", TYPES, ids=IDS)
@pytest.mark.parametrize("m,c,k", [(16, 4100, 500), (3, 25088, 300), (5, 25088, 300), (16, 9000, 64), (8, 8192, 4000)])
def test_more_than_64_kb_of_rows(F, m, c, k, xt):  # noqa: F811
    """Rows that are staged in up to 144 KB of LDS, in one turn or several, with each group size after the other."""
    for group in (128, 32, 64):
        check(F, m, c, k, xt, group, group != 64, group == 32)


# sizes that between them are served by every kernel and shape there is, with their columns divided and not (a test on the CPU asks the choice)
CASES = [(1, 44, 34), (7, 42, 34), (1, 9304, 37), (3, 8341, 35), (17, 4161, 43), (20, 8122, 53), (18, 49, 42), (17, 135, 46), (33, 169, 8722), (33, 8911, 12512), (38, 7210, 1041),
         (961, 41, 6411), (176, 5292, 2759), (9173, 401, 134), (39, 15106, 8810), (3623, 63697, 143)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("xt,rows", [(torch.float32, False), (torch.float16, False), (torch.bfloat16, False), (torch.int8, False), (torch.int8, True)],
                         ids=["f32", "f16", "bf16", "i8-groups", "i8-rows"])
@pytest.mark.parametrize("m,c,k", CASES)
def test_every_kernel(F, m, c, k, xt, rows, group):  # noqa: F811
    check(F, m, c, k, xt, group, (m + group) % 3 > 0, rows, ("apart", "odd"), ("no room",))


# more than 16 rows (fp32: five), few weight rows, many columns
@pytest.mark.parametrize("xt,rows", [(torch.float32, False), (torch.float16, False), (torch.bfloat16, False), (torch.int8, False), (torch.int8, True)],
                         ids=["f32", "f16", "bf16", "i8-groups", "i8-rows"])
@pytest.mark.parametrize("m,c,k", [(17, 9000, 43), (64, 20001, 300), (38, 7210, 1041), (3623, 63697, 143)])
def test_scratch_is_used(F, m, c, k, xt, rows):  # noqa: F811
    for group in (32, 64, 128):
        check(F, m, c, k, xt, group, True, rows, ("odd",), ("no room", "room"))
