"""Products with 4-bit weights at the sizes that take each shape of the kernels, bit for bit on integers: few work-groups and many, blocks divided over
waves and over work-groups (with scratch, with less and with none), rows of x aligned and not, one column and one weight row, more rows than a launch
holds; the widest integers; weights whose scales are not finite; and norm, 8 bits and product captured as one."""
import ctypes

import pytest
import torch

from test_gpu_q4 import F, FLOATS, apart, dense, ints, packed, rng, weights, wide  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = FLOATS + [torch.int8]


def problem(F, m, c, k, xt, group=128, zeros=True, seed=0):
    """Handle, x, its scales and the exact result: sums of multiples of 1/4 that 32 bits hold (x in -1..1, at most 15 * 2 a product)."""
    g = rng(seed + m + c + k)
    q, s, z = weights(g, k, c, group, zeros, powers=True)
    h = F.q4_import(packed(q), s, z, group=group, c=c)
    x = ints(g, -1, 2, m, c).to(xt)
    xs = None
    if xt == torch.int8:
        xs = torch.exp2(ints(g, -1, 1, m, (c + group - 1) // group).float()) if seed % 2 == 0 else torch.exp2(ints(g, -1, 1, m).float())
    x64 = x.double() * (1 if xs is None else (wide(xs, group, c) if xs.dim() == 2 else xs.double()[:, None]))
    return h, x, xs, x64 @ dense(q, s, z, group)[0].t()


# rows, columns, weight rows: the tiles of 16 and 8 bits from 32 x 32 in eight sets to 128 x 128 in one, then divided columns of fp32
SIZES = [(40, 1100, 1000), (100, 1100, 4100), (200, 1024, 4096), (700, 1024, 4096), (650, 1100, 4000), (1000, 520, 2100), (900, 300, 8200), (500, 1100, 4096), (1900, 1100, 4090),
         (32, 8192, 640), (6, 5000, 90), (16, 4100, 400), (120, 6000, 100), (200, 1, 70), (200, 70, 1), (40, 1, 1)]


@pytest.mark.parametrize("xt", TYPES, ids=["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("m,c,k", SIZES)
def test_every_shape(F, m, c, k, xt):  # noqa: F811
    case = SIZES.index((m, c, k))
    h, x, xs, want = problem(F, m, c, k, xt, (128, 64, 32)[case % 3], case % 2 == 0, case)
    yt = torch.float32
    assert torch.equal(F.linear_q4(h, x, x_scale=xs, out_dtype=yt).double(), want)
    e = 16 // x.element_size()
    assert torch.equal(F.linear_q4(h, apart(x, (-c) % e + e), x_scale=xs, out_dtype=yt).double(), want)
    assert torch.equal(F.linear_q4(h, apart(x, 1, 3), x_scale=xs, out_dtype=yt).double(), want)


@pytest.mark.parametrize("m,c,k", [(6, 5000, 90), (32, 8192, 640), (120, 6000, 100), (300, 2100, 1000)])
def test_scratch(F, m, c, k):  # noqa: F811
    """A call with the scratch it asks for writes no byte behind it; with less, or none, the result is the same."""
    h, x, _, want = problem(F, m, c, k, torch.float32)
    L, ll = F.lib(), ctypes.c_longlong
    L.fscnn_linear_q4_workspace.restype = ll
    need = L.fscnn_linear_q4_workspace(h.handle, 0, m)
    assert need >= 0 and need % 4 == 0
    ws = torch.full((need // 4 + 65,), 7.0, device="cuda")[1:]      # (4 bytes aligned, no more)
    for size in (need, need - 4, 4, 0):
        y = torch.zeros(m, k, device="cuda")
        st = L.fscnn_linear_q4(h.handle, ctypes.c_void_p(x.data_ptr()), 0, ll(c), None, 1, m, c, None, ctypes.c_float(1.0), ctypes.c_void_p(y.data_ptr()), 0, ll(k),
                               ctypes.c_void_p(ws.data_ptr()) if size > 0 else None, ll(max(size, 0)), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0 and torch.equal(y.double(), want) and bool((ws[need // 4:] == 7).all())


@pytest.mark.parametrize("rows", [0, 1], ids=["groups", "rows"])
@pytest.mark.parametrize("xt", TYPES[1:], ids=["f16", "bf16", "i8"])
@pytest.mark.parametrize("m,c,k", [(64, 20001, 300), (20, 9000, 512), (200, 8200, 250), (17, 4096, 256), (130, 1100, 40)])
def test_scratch_of_narrow_rows(F, m, c, k, xt, rows):  # noqa: F811
    """The same of rows in 16 and 8 bits, which have scales by group or by row."""
    h, x, xs, want = problem(F, m, c, k, xt, 128, True, rows)
    L, ll, t = F.lib(), ctypes.c_longlong, F._DTYPES[xt]
    L.fscnn_linear_q4_workspace.restype = ll
    need = L.fscnn_linear_q4_workspace(h.handle, t, m)
    assert need >= 0 and need % 64 == 0
    ws = torch.full((need // 4 + 65,), 7.0, device="cuda")[1:]
    for size in (need, need - 4, 0):
        y = torch.zeros(m, k, device="cuda")
        st = L.fscnn_linear_q4(h.handle, ctypes.c_void_p(x.data_ptr()), t, ll(c), ctypes.c_void_p(xs.data_ptr()) if xs is not None else None,
                               xs.numel() // m if xs is not None else 1, m, c, None, ctypes.c_float(1.0), ctypes.c_void_p(y.data_ptr()), 0, ll(k),
                               ctypes.c_void_p(ws.data_ptr()) if size > 0 else None, ll(max(size, 0)), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0 and torch.equal(y.double(), want) and bool((ws[need // 4:] == 7).all())


@pytest.mark.parametrize("xt", TYPES, ids=["f32", "f16", "bf16", "i8"])
def test_more_rows_than_a_launch_holds(F, xt):  # noqa: F811
    m, c, k = (1 << 18) + 77, 40, 24
    for seed in (0, 1):
        h, x, xs, want = problem(F, m, c, k, xt, 32, True, seed)
        assert torch.equal(F.linear_q4(h, x, x_scale=xs, out_dtype=torch.float32).double(), want)
        assert torch.equal(F.linear_q4(h, apart(x, 3, 1), x_scale=xs, out_dtype=torch.float32).double(), want)


@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_widest_integers(F, m):  # noqa: F811
    """x of -128 and 127 against differences of -15 and 15: a group's sum is at most 128 * 128 * 15 and exact; eight groups stay below 2^24."""
    k, c = 70, 1024
    for code, zero in ((0, 15), (15, 0)):
        codes = torch.full((k, c // 2), code * 17, dtype=torch.uint8, device="cuda")
        h = F.q4_import(codes, torch.ones(k, c // 128, dtype=torch.float16, device="cuda"), torch.full((k, c // 128), zero, dtype=torch.uint8, device="cuda"), group=128)
        x = torch.full((m, c), -128, dtype=torch.int8, device="cuda")
        x[::2] = 127
        want = (x.double().sum(1, keepdim=True) * (code - zero)).expand(m, k)
        for xs in (torch.ones(m, device="cuda"), torch.ones(m, c // 128, device="cuda")):
            assert torch.equal(F.linear_q4(h, x, x_scale=xs).double(), want)


@pytest.mark.parametrize("xt", TYPES, ids=["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("m", [1, 4, 16, 50, 300])
def test_scales_that_are_not_finite_stay_in_their_weight_row(F, m, xt):  # noqa: F811
    g = rng(m)
    k, c = 150, 260
    q, s, z = weights(g, k, c, 64, True, powers=True)
    x = ints(g, 1, 3, m, c).to(xt)
    xs = torch.ones(m, device="cuda") if xt == torch.int8 else None
    want = F.linear_q4(F.q4_import(packed(q), s, z, group=64, c=c), x, x_scale=xs, out_dtype=torch.float32)
    s[17, 4], s[149, 0] = float("nan"), float("inf")
    s[3] = 0
    s[4] *= -1
    got = F.linear_q4(F.q4_import(packed(q), s, z, group=64, c=c), x, x_scale=xs, out_dtype=torch.float32)
    assert not bool(torch.isfinite(got[:, [17, 149]]).any()) and not got[:, 3].any() and torch.equal(got[:, 4], -want[:, 4])
    keep = [i for i in range(k) if i not in (3, 4, 17, 149)]
    assert torch.equal(got[:, keep], want[:, keep])


@pytest.mark.parametrize("m", [1, 20, 300])
def test_a_layer_captured(F, m):  # noqa: F811
    """Residual, norm, 8 bits and product in one graph, its inputs changed between the replays; eager calls beside it."""
    g = rng(m)
    d, k = 640, 330
    q, s, z = weights(g, k, d, 64, True)
    h = F.q4_import(packed(q), s, z, group=64, c=d)
    x, r = (torch.zeros(m, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")

    def layer():
        q8, sc, out = F.rms_norm_q8(x, w, 1e-5, residual=r, group=64)
        return F.linear_q4(h, q8, x_scale=sc, out_dtype=torch.bfloat16), out

    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, out = layer()
    for _ in range(3):
        x.copy_(torch.randn(m, d, generator=g, device="cuda"))
        r.copy_(torch.randn(m, d, generator=g, device="cuda"))
        graph.replay()
        y2, out2 = layer()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(out, out2) and bool(y.any())


@pytest.mark.parametrize("kind", ["relu", "positive"])
@pytest.mark.parametrize("m", [1, 4, 8, 14, 40, 200])
def test_precision_of_values_that_are_not_negative(F, m, kind):  # noqa: F811
    """fp32 rows without negative values, whose sums with codes are far larger than with weights.  Per group 24 additions in the matrix cores (three
    parts, eight steps), each off by at most a step of the sum so far, 2^-23 of it, if it cuts; 32 groups are added with half a step each.  Sums of
    weights around zero grow like a root, their mean size on the way is 2/3 of the last one: (24 + 32 / 2) * 2/3 * 2^-23 = 27 * 2^-23 of the
    result, in the mean over the outputs, had every addition erred to the same side; they do not."""
    c, k = 4096, 512
    g = rng(m)
    wd = torch.randn(k, c, generator=g, device="cuda") / 64
    h = F.q4_compress(wd, 128, True)
    codes, scales, zeros = (t.cuda() for t in F.q4_export(h))
    w = dense(torch.stack([codes & 15, codes >> 4], 2).view(k, -1), scales, zeros, 128)[0]
    x = torch.randn(m, c, generator=g, device="cuda")
    x = x.clamp(min=0) if kind == "relu" else x.abs() + 3
    want = x.double() @ w.t()
    got = F.linear_q4(h, x).double()
    assert float((got - want).norm()) <= 27 * 2.0 ** -23 * float(want.norm())


@pytest.mark.parametrize("xt", TYPES, ids=["f32", "f16", "bf16", "i8"])
@pytest.mark.parametrize("m", [1, 5, 12, 40])
def test_the_longest_rows(F, m, xt):  # noqa: F811
    """2^20 columns, the most there may be: sums stay below 2^22 (a random walk of 2^20 steps of at most 30)."""
    h, x, xs, want = problem(F, m, 1 << 20, 20, xt, 128, True, 1)
    assert float(want.abs().max()) < 2 ** 22
    assert torch.equal(F.linear_q4(h, x, x_scale=xs, out_dtype=torch.float32).double(), want)


def test_codes_at_any_byte(F):  # noqa: F811
    g = rng(4)
    for k, c in ((33, 129), (40, 1024), (17, 7), (20, 8)):
        q, s, z = weights(g, k, c, 32, True)
        p = packed(q)
        want = F.q4_export(F.q4_import(p, s, z, group=32, c=c))
        for off in (1, 2, 3):
            buf = torch.full((p.numel() + off + 8,), 255, dtype=torch.uint8, device="cuda")
            view = buf[off:off + p.numel()].view(p.shape)
            view.copy_(p)
            assert all(torch.equal(a, b) for a, b in zip(F.q4_export(F.q4_import(view, s, z, group=32, c=c)), want))


def test_threads(F):  # noqa: F811
    """Four threads, each on a stream of its own, with one set of weights: products with and without scratch, and the norm."""
    import threading
    g = rng(6)
    d, k = 2048, 96
    q, s, z = weights(g, k, d, 128, True)
    h = F.q4_import(packed(q), s, z, group=128, c=d)
    xs = [torch.randn(m, d, generator=g, device="cuda") for m in (1, 12, 60, 130)]
    w = torch.ones(d, device="cuda")
    layer = lambda x: (F.linear_q4(h, x), F.linear_q4(h, x.half()), F.rms_norm(x, w), *F.rms_norm_q8(x, w, group=64))
    want = [layer(x) for x in xs]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for _ in range(20):
                    got = layer(xs[i])
                    st.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        bad.append(i)
        except Exception as e:
            bad.append(e)

    ts = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert not bad


@pytest.mark.parametrize("xt", TYPES, ids=["f32", "f16", "bf16", "i8"])
def test_the_binding_s_scratch_has_the_bytes_it_names(F, xt, monkeypatch):  # noqa: F811
    """Nothing is launched: a stand-in for the native call looks at what it is handed."""
    m, c, k = 64, 20000, 300
    h = F.q4_import(torch.zeros(k, c // 2, dtype=torch.uint8, device="cuda"), torch.ones(k, (c + 127) // 128, dtype=torch.float16, device="cuda"))
    native = F._native()
    need = native.linear_q4_workspace(h.address, F._DTYPES[xt], m)
    assert need > 0
    seen = []

    class Stand:
        linear_q4_workspace = staticmethod(native.linear_q4_workspace)

        @staticmethod
        def linear_q4(*args):
            seen.append((args[13], args[14], torch.cuda.memory_stats()["requested_bytes.all.allocated"]))
            return 0

    x, out = torch.zeros(m, c, dtype=xt, device="cuda"), torch.empty(m, k, dtype=torch.float32, device="cuda")
    scale = torch.ones(m, device="cuda") if xt == torch.int8 else None
    monkeypatch.setattr(F, "_nat", Stand)
    before = torch.cuda.memory_stats()["requested_bytes.all.allocated"]
    F.linear_q4(h, x, x_scale=scale, out=out)
    assert len(seen) == 1 and seen[0][0] and seen[0][1] == need and seen[0][2] - before >= need
