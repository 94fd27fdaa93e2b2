"""Which kernel serves a product with 4-bit weights (csrc/q4_choice.h), compiled and asked on the CPU."""
import math
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include "q4_choice.h"
#include <cstdio>
using namespace fscnn;
int main()                                     // x_type M K C aligned room  ->  kernel waves shape parts us
{
    int t, M, K, C, aligned, room;
    while (std::scanf("%d %d %d %d %d %d", &t, &M, &K, &C, &aligned, &room) == 6) {
        const int parts = room ? q4_parts(t, M, K, C) : 1, blocks = (C + 127) / 128, rows = M < kQ4LaunchRows ? M : kQ4LaunchRows;
        const Q4Choice c = t == FSCNN_F32 ? f32_choice((K + 15LL) / 16, blocks, rows, parts) : narrow_choice(t == FSCNN_I8, rows, K, blocks, parts, aligned);
        std::printf("%d %d %d %d %g\n", c.kernel, c.waves, c.shape, parts, c.us);
    }
}
"""
F32, F16, BF16, I8 = range(4)
ROWS, STAGED, TILES = range(3)


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("choice")
    (d / "choice.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2212_08815_amd", "csrc"),
                    str(d / "choice.cpp"), "-o", str(d / "choice")], check=True)

    def f(cases):
        r = subprocess.run([str(d / "choice")], input="\n".join(" ".join(map(str, map(int, c))) for c in cases), capture_output=True, text=True, check=True)
        return [(int(a[0]), int(a[1]), int(a[2]), int(a[3]), float(a[4])) for a in (line.split() for line in r.stdout.splitlines())]
    return f


def test_few_columns_of_fp32(ask):
    """Fewer than four blocks of columns: the cheaper of a wave's own rows and tiles, as with more (16 rows to 60000 of 384: 20.2 us the former, 10.5
    tiles); tiles of 32 rows for more rows."""
    sizes = [(6, 60000, 384), (16, 60000, 384), (16, 30000, 256), (10, 60000, 128), (6, 4096, 300), (16, 4096, 384), (12, 12288, 384), (17, 60000, 384), (4096, 16384, 384),
             (900, 8200, 300), (40, 1000, 1)]
    want = [TILES] * 4 + [ROWS] * 3 + [TILES] * 4
    for room in (0, 1):
        got = ask([(F32, m, k, c, 1, room) for m, k, c in sizes])
        assert [c[0] for c in got] == want and all(c[2] == 32 for c in got if c[0] == TILES) and all(c[3] == 1 and c[4] < 1e4 for c in got)


def served(ask, sizes):
    """What serves calls of these sizes, in every type, with their rows 16 bytes aligned and not, with scratch and without; and into how many parts columns
    are divided."""
    calls = [(t, m, k, c, al, room) for m, c, k in sizes for t in (F32, F16, I8) for al in ((0, 1) if t != F32 else (1,)) for room in (0, 1)]
    out = set()
    for (t, m, k, c, al, room), (kernel, waves, shape, parts, _) in zip(calls, ask(calls)):
        out |= {(t, kernel, waves, shape, parts > 1, al), (t, parts)}
    return out


def test_the_gpu_tests_reach_every_kernel(ask):
    """What the choice gives for 50 thousand sizes of all magnitudes is run by tests/test_gpu_q4_groups.py, there with every group size and way of scaling."""
    from test_gpu_q4_groups import CASES
    r = random.Random(3)
    any_size = lambda hi: int(round(math.exp(r.uniform(0, math.log(hi)))))
    assert served(ask, [(any_size(20000), any_size(1 << 20), any_size(60000)) for _ in range(50000)]) <= served(ask, CASES)


LAUNCHES = r"""
#include "q4_choice.h"
#include <cstdio>
using namespace fscnn;
int main()                                     // K -> rows of x a launch
{
    int K;
    std::printf("%d\n", kQ4MostRows);
    while (std::scanf("%d", &K) == 1) std::printf("%d\n", q4_launch_rows(K));
}
"""


def test_a_launch_holds_its_threads(ask, tmp_path):
    """Fewer than 2^32 threads for any number of rows of x and of weights: tiles by the choice's shapes, 16 weight rows a work-group where x has few rows."""
    (tmp_path / "launch.cpp").write_text(LAUNCHES)
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2212_08815_amd", "csrc"), str(tmp_path / "launch.cpp"),
                    "-o", str(tmp_path / "launch")], check=True)
    r = random.Random(5)
    most = 2 ** 27 - 16
    ks = [1, 32768, 32769, 262145, 1 << 20, most - 1, most] + [int(2 ** r.uniform(0, 27)) for _ in range(300)]
    ks = [min(k, most) for k in ks]
    out = subprocess.run([str(tmp_path / "launch")], input=" ".join(map(str, ks)), capture_output=True, text=True, check=True).stdout.split()
    assert int(out[0]) == most
    tiles = {F32: {32: (32, 256, 512), 64: (64, 256, 512)},
             F16: dict(enumerate([(32, 32, 512), (32, 64, 512), (64, 128, 512), (64, 128, 256), (128, 128, 256), (64, 64, 512), (96, 128, 512)]))}
    tiles[I8] = tiles[F16]
    up = lambda a, b: -(-a // b)
    for k, rows in zip(ks, map(int, out[1:])):
        assert 32 <= rows <= 1 << 18 and (k > 30000 or rows == 1 << 18)
        calls = [(t, m, k, c, al, 1) for t in tiles for al in (0, 1) for m in (1, 5, 16, rows // 2 + 1, rows) for c in (1, 128, 600, 5000)]
        for (t, m, *_), (kernel, waves, shape, parts, _) in zip(calls, ask(calls)):
            if kernel == TILES:
                a, b, threads = tiles[t][shape]
                n = up(m, a) * up(k, b) * threads      # (parts are the grid's second dimension)
            else:
                n = up(k, 16) * waves * 64
            assert n < 2 ** 32
