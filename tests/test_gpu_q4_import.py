"""q4_import and q4_compress wait for their own stream and for nothing else."""
import ctypes

import pytest
import torch

from test_gpu_q4 import F, ints, packed, rng, weights  # noqa: F401

pytestmark = pytest.mark.gpu


def test_other_streams_are_not_waited_for(F):  # noqa: F811
    """A stream that the default one waits for has a tenth of a second of work; codes are imported, and weights compressed, beside it."""
    hip = ctypes.CDLL("libamdhip64.so")
    raw = ctypes.c_void_p()
    assert hip.hipStreamCreate(ctypes.byref(raw)) == 0
    busy, own = torch.cuda.ExternalStream(raw.value), torch.cuda.Stream()
    g = rng(1)
    q, s, z = weights(g, 200, 1000, 64, True)
    p, w = packed(q), torch.randn(200, 1000, generator=g, device="cuda")
    big = torch.zeros(1 << 29, device="cuda")
    with torch.cuda.stream(own):
        F.q4_import(p, s, z, group=64, c=1000)
        F.q4_compress(w, 64, True)
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        for _ in range(100):                           # a millisecond each
            big.add_(1.0)
    with torch.cuda.stream(own):
        h = F.q4_import(p, s, z, group=64, c=1000)
        c = F.q4_compress(w, 64, True)
    beside = not busy.query()
    torch.cuda.synchronize()
    assert hip.hipStreamDestroy(raw) == 0
    assert beside
    assert torch.equal(F.q4_export(h)[2], z.cpu()) and F.q4_export(c)[0].any()
    # and a zero point above 15 is found
    z[199, 15] = 16
    with torch.cuda.stream(own), pytest.raises(F.FscnnError) as e:
        F.q4_import(p, s, z, group=64, c=1000)
    assert e.value.status == 4
