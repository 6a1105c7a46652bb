"""Softmax weights far below the largest one: a first row that has nearly all the weight and a value of zero leaves an output that
the small weights alone make, so that every bit that the 16-bit parts of a weight lose shows."""
import math

import pytest
import torch

import paper_2406_02069_b200 as pkv
from cache_oracle import TYPES, attend
from test_gpu_cache_attention import Data

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = float(torch.tensor(math.log(2.0), dtype=torch.float32))      # logits in powers of two: times log2(e) it is 1 in fp32


def sink(heads, d, dtype, rows, below):
    """Row 0: logit 0, value 0.  The others: logit f - below (in powers of two) for head g's f = (2 g + 1) / 16, values of one sign (so that errors
    that all rows share add up) between 0.5 and 1."""
    t = TYPES[dtype]
    group, kv = heads[0] // heads[1], heads[1]
    g = torch.Generator().manual_seed(rows + below)
    q = torch.zeros(1, heads[0], d)
    q[..., 0] = 1.0
    q[..., 1] = ((2 * (torch.arange(heads[0]) % group) + 1) % 16) / 16
    k = torch.zeros(kv, rows, d)
    k[:, 1:, 0], k[:, 1:, 1] = -below, 1.0
    v = torch.rand(kv, rows, d, generator=g) / 2 + 0.5
    v[:, 0] = 0
    return q.to(t), k.to(t), v.to(t)


def tolerance(rows, exponent):
    """Relative to the sum of small weights times |V|.  A weight: the approximate power of two is off by 2^-22 at most, the parts
    leave 2^-24, and where the exponent is rounded (the product with the scale and the scale itself, a step of 2^-24 each, times
    the logarithm of two) 2 * 2^-24 ln 2 * exponent.  The sum of the weights: 4 roundings.  The weighted sum: 16 products of a
    step cut off at 2^-23 of their sum at most, three parts joined, four warps (eight in fp32), then a rounding for every tile of
    64 rows twice over (added up, joined): 14 + tiles * 2 roundings of 2^-24."""
    tiles = -(-rows // 64)
    return 2.0 ** -22 + 2.0 ** -24 + 2 * 2.0 ** -24 * math.log(2) * exponent + (4 + 2 + 14 + 2 * tiles) * 2.0 ** -24


@pytest.mark.parametrize("below", [17, 21, 27])
@pytest.mark.parametrize("rows", [64, 700])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("heads,d", [((2, 2), 64), ((8, 2), 128), ((8, 1), 128), ((12, 1), 64)])
def test_small_weights_keep_their_bits(heads, d, dtype, rows, below):
    x = Data(heads, d, dtype, 16, [rows])
    q, k, v = sink(heads, d, dtype, rows, below)
    x.q, x.k, x.v = q, [k], [v]
    x.fill()
    out, lse = x.run(scale=SCALE)
    group = heads[0] // heads[1]
    bound = tolerance(rows, 0)                                       # (dot products and their exponents are exact here)
    for h in range(heads[1]):
        hq = slice(h * group, (h + 1) * group)
        want, want_lse, size = attend(q[0, hq], k[h], v[h], scale=SCALE)
        off = (out[0, hq].double() - want).abs() / size
        assert float(off.max()) <= bound, (h, float(off.max()), bound)
        assert torch.all((lse[0, hq].double() - want_lse).abs() <= bound)
