"""The 8-bit cache at the ends of its ranges: infinities beside the largest magnitudes, sums and logits near the largest numbers, queries of very
unequal elements, slabs that reach beyond their buffers, range lists that make no sense."""
import numpy as np
import pytest
import torch

import oracle
from q8_common import DT, Cache, bf16, random_slab
from test_gpu_q8 import B, FORMATS, attend, check_attention, filled, queries, same  # noqa: F401

pytestmark = pytest.mark.gpu
LARGEST = float(torch.finfo(torch.bfloat16).max)


# ------------------------------------------------------------------ infinities
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("block", [16, 128])
def test_infinities_beside_the_largest_magnitude(B, fmt, paged, block):
    """Stored as the largest codes of their signs under the largest scale there is too: packed, and joining a block that has it (a row at a time,
    and more rows than go without tiles)."""
    r = np.random.default_rng(4)
    first = r.normal(0, 1, (21, 128))
    first[3, :5] = LARGEST, np.inf, -np.inf, -LARGEST, np.nan
    first[20, 7] = -LARGEST
    later = []
    for n in (1, 4, 5, 30):
        x = r.normal(0, 1, (n, 128))
        x[n - 1, 9:12] = np.inf, -np.inf, LARGEST / 2
        x[0, 100] = -np.inf
        later.append(bf16(x))
    first = bf16(first)
    c = Cache(B, [[21]], [200], 1, fmt, block, paged, 1)
    src = torch.zeros(c.rows16, 128, dtype=torch.bfloat16)
    src[:21] = first
    B.skipkv_pack_q8(c.shape, c.cache, src.cuda(), src.cuda(), c.kv_len, c.ws)
    torch.cuda.synchronize()
    assert c.status() == 8
    codes, scale = np.zeros((200, 128), np.uint8), np.zeros(-(-200 // block))
    n = oracle.q8_append(codes, scale, 0, first.double().numpy(), block, fmt)
    assert scale[0] == 2.0 ** (122 if fmt == "int8" else 120)
    same(c, 0, n, [codes] * 2, [scale] * 2)
    a, b = c.kv_len.clone(), torch.zeros_like(c.kv_len)
    for x in later:
        rows = x.view(-1, 1, 128).cuda()
        B.skipkv_append_q8(c.shape, c.cache, rows, rows, torch.tensor([0, len(x)], dtype=torch.int32).cuda(), len(x), a, b, c.ws)
        torch.cuda.synchronize()
        assert c.status() == 8
        n = oracle.q8_append(codes, scale, n, x.double().numpy(), block, fmt)
        assert b.item() == n
        same(c, 0, n, [codes] * 2, [scale] * 2)
        a, b = b, a
