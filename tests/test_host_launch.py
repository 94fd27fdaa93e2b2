"""The library's launches, as its symbols show them."""
import os
import re


def test_each_staged_kernel_has_its_lds_asked_for():
    """A kernel that may want more than 64 KB of LDS has the limit raised once, by a static of its own: as many of these (their guards) as there are
    kernels, or one that is not launched first never has it raised."""
    from paper_2212_08815_amd import fscnn
    if not os.path.exists(fscnn.LIB_PATH):
        from paper_2212_08815_amd import build
        build.build()
    with open(fscnn.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"_Z[A-Za-z0-9_]{8,}", f.read()))
    kernels = {n for n in names if b"__device_stub__staged_kernel" in n}
    guards = {n for n in names if n.startswith(b"_ZGVZ") and b"launch_staged" in n and n.endswith(b"attr")}
    assert len(kernels) == 24 and len(guards) == len(kernels)
