"""Decode attention over the compact cache where one row has nearly all the weight and a value of zero: what is left of the output
is made by weights far below the largest one, and every bit that their 16-bit parts lose shows."""
import math

import pytest
import torch

import paper_2406_02069_b200 as pkv

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("below", [14, 24, 27])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("group,d,rows", [(1, 128, 64), (4, 64, 200), (6, 128, 1000)])
def test_small_weights_keep_their_bits(group, d, rows, dtype, below):
    t = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    cfg = pkv.make_config(num_layers=1, num_q_heads=2 * group, num_kv_heads=2, head_dim=d, window=1, pool_kernel=1, dtype=dtype, avg_budget=1)
    lens, kl = [5000], rows - 1
    assert pkv.kept_count(cfg, kl, lens[0]) == rows
    g = torch.Generator().manual_seed(rows + below)
    q = torch.zeros(1, 2 * group, d)
    q[..., 0] = math.log(2) * math.sqrt(d)
    q[..., 1] = math.log(2) * math.sqrt(d) * (2 * torch.arange(2 * group) + 1) / 16
    k = torch.zeros(2, rows, d)
    k[:, 1:, 0], k[:, 1:, 1] = -below, 1.0
    v = torch.rand(2, rows, d, generator=g) / 2 + 0.5
    v[:, 0] = 0
    q, k, v = q.to(t), k.to(t), v.to(t)
    out = torch.full((1, 2 * group, d), 7.0, device=DEV)
    pkv.decode_attention(cfg, q.to(DEV), k.view(-1, d).to(DEV), v.view(-1, d).to(DEV), lens, kl, out)
    # The exponent x: two products added (cut off at 2^-23 of their sum, or a rounding each), the factor log2(e) / sqrt(d) and its
    # product: 5 steps of 2^-24 of |x| < below + 1.  A weight: the approximate power of two 2^-22, the parts 2^-24.  The sum of the
    # weights 6 roundings; the weighted one: 16 products of a step, three parts, warps, CTAs and one addition a step of 16 rows.
    bound = 5 * 2.0 ** -24 * math.log(2) * (below + 1) + 2.0 ** -22 + 2.0 ** -24 + (6 + 24 + rows / 16) * 2.0 ** -24
    for h in range(2):
        hq = slice(h * group, (h + 1) * group)
        x = q[0, hq].double() @ k[h].double().T / math.sqrt(d)
        w = torch.softmax(x, -1)
        want = w @ v[h].double()
        off = (out[0, hq].cpu().double() - want).abs() / want
        assert float(off.max()) <= bound, (h, float(off.max()), bound)
