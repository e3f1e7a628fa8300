"""Contexts on streams other than the default one, from their first call on:
the accumulators of the fused row binding are cleared in the stream's own
order, so that layers proven at once on two streams match the oracle."""
import numpy as np
import pytest
import torch

from helpers import diff_transcripts
from oracle import oracle as orc
from paper_2505_17623_amd import inputs

pytestmark = pytest.mark.gpu


def test_first_layers_on_side_streams():
    from paper_2505_17623_amd import ra
    rng = np.random.default_rng(1)
    n, m, k = 16, 512, 16
    A, B = (rng.integers(-500, 500, s).astype(np.int16) for s in ((n, m), (m, k)))
    dA, dB = torch.from_numpy(A).cuda(), torch.from_numpy(B).cuda()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(4):
        chal = inputs.xorshift64_stream(70 + rep, 1000)
        want = orc.prove_layer(A, B, 8, True, 0, chal, 0)
        got = []
        for st in streams:
            with torch.cuda.stream(st):
                ctx = ra.Context(chal, stream=st, deferred=True)
                got.append((ctx, ra.prove_layer(ctx, dA, dB, 8, True, t=want["t"])))
        for ctx, res in got:
            ctx.sync()
            assert not diff_transcripts(res["transcript"], want)
