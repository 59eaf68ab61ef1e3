"""A half-precision output is a value nearest to the fp32 output: whatever the output's type, the sums take the same order.

The result may be rounded from the fp32 value y = fl(x) or from the exact product x: where y lies halfway between two half-precision values these
are the two, and elsewhere they are equal, since the halves are fp32 values, which no rounding to fp32 passes.  So the distance to y is the
least there is, without a tolerance."""
import pytest
import torch

from paper_1804_08066_amd import mqgrad as mq
from test_gpu_embedding import BF16, DEV, F16, F32, TYPES, matrix, some_tokens

pytestmark = pytest.mark.gpu


def nearest(short, long):
    least = (long.to(short.dtype).double() - long.double()).abs()
    return torch.equal((short.double() - long.double()).abs(), least)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("out", [F16, BF16], ids=str)
@pytest.mark.parametrize("count", [90, 3000, 9000, 40_000])
def test_gradient(count, out, accumulate):
    for dim in (3, 72, 520):
        g, ids = matrix(count, dim, 1, BF16), some_tokens("text", count, 400).to(DEV)
        old = matrix(400, dim, 2, out)
        short, long = old.clone(), old.to(F32)
        for t in (short, long):
            mq.mqg_embedding_grad(g, ids, 400, scale=-0.3, out=t, accumulate=accumulate)
        assert nearest(short, long)


@pytest.mark.parametrize("out", [F16, BF16], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_lookup_and_clipping(dtype, out):
    table, ids = matrix(50, 77, 3, dtype), some_tokens("shards", 300, 50).to(DEV)
    rows = [mq.mqg_embedding(table, ids, scale=0.7, out=torch.empty(300, 77, dtype=t, device=DEV)) for t in (out, F32)]
    assert nearest(*rows)
    outputs = [torch.empty(50, 77, dtype=t, device=DEV) for t in (out, F32)]
    for o in outputs:
        mq.mqg_clip_global_norm([table], 3.0, outputs=[o])
    assert nearest(*outputs)
