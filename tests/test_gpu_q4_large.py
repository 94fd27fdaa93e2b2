"""More weights than a launch has threads for."""
import pytest
import torch

from test_gpu_q4 import F, dense, ints, rng  # noqa: F401

pytestmark = pytest.mark.gpu


def test_more_than_2_to_the_35_weights(F):  # noqa: F811
    """33000 x 2^20: codes and scales in, products with rows from both ends, codes and scales back from compressed ones."""
    k, c, group = 33000, 1 << 20, 128
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("needs 150 GB")
    g = rng(2)
    codes = torch.empty(k, c // 2, dtype=torch.uint8, device="cuda")
    for lo in range(0, k, 3000):
        codes[lo:lo + 3000] = torch.randint(0, 256, codes[lo:lo + 3000].shape, generator=g, device="cuda", dtype=torch.uint8)
    s = torch.exp2(ints(g, -2, 2, k, c // group).float()).half()
    h = F.q4_import(codes, s, group=group)
    x = ints(g, -1, 2, 2, c).half()
    got = F.linear_q4(h, x, out_dtype=torch.float32)
    for lo in (0, 16384, k - 64):
        q = torch.stack([codes[lo:lo + 64] & 15, codes[lo:lo + 64] >> 4], 2).view(64, -1)
        assert torch.equal(got[:, lo:lo + 64], (x.double() @ dense(q, s[lo:lo + 64], None, group)[0].t()).float())
    back = F.q4_export(h)
    assert torch.equal(back[0][-1], codes[-1].cpu()) and torch.equal(back[0][0], codes[0].cpu()) and torch.equal(back[1], s.cpu())
    h.destroy()
    del codes, back
    w = torch.ones(1, c, device="cuda").half().expand(k, c).contiguous()
    w[-1] = -2
    h = F.q4_compress(w, group)
    y = F.linear_q4(h, torch.ones(1, c, device="cuda").half(), out_dtype=torch.float32)[0]
    assert bool((y[:-1] == y[0]).all()) and float(y[-1]) == -2 * float(y[0])
