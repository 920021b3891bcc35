"""si_cache_append with two tokens for one place: every element is that of one of them, and nothing else changes."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from attention_reference import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [si.SI_KV_BF16, si.SI_KV_E4M3])
@pytest.mark.parametrize("n,first", [(2, 5), (40, 0), (70, 3)])
def test_a_place_named_twice(kind, n, first):
    """Tokens first .. first + n - 1 of sequence 0, twice, and one place of sequence 1."""
    kv, d, page = 3, 128, 128
    c = Cache(kind, 3, page, 2, 1, 1, kv, d, seed=n)
    c.table[0, 0], c.table[1, 0] = 2, 0
    T = 2 * n + 1
    pos = torch.tensor(list(range(first, first + n)) * 2 + [9], dtype=torch.int32, device="cuda")
    seq = torch.tensor([0] * (2 * n) + [1], dtype=torch.int32, device="cuda")
    kvs = torch.randint(-8, 9, (T, 2, kv, d), generator=torch.Generator().manual_seed(n)).to(torch.bfloat16).cuda()  # (integers: e4m3 holds them)
    before = c.bits().copy()
    row = 2 * kv * d
    si.si_cache_append(c.desc, 0, si.si_append_t(k=kvs.data_ptr(), v=kvs.data_ptr() + 2 * kv * d, seq=seq.data_ptr(), pos=pos.data_ptr(), k_stride=row, v_stride=row, n_tokens=T),
                       torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    x, val = kvs.double().cpu().numpy(), c.values()
    ik, iv = c.places(np.arange(first, first + n))
    same = np.ones(before.shape, bool)
    for h in range(kv):
        for which, at in ((0, ik), (1, iv)):
            got = val[2, 0, which, h][at]
            assert np.all((got == x[:n, which, h]) | (got == x[n:2 * n, which, h]))
            same[2, 0, which, h][at] = False
            one = c.places([9])[which][0]
            assert np.array_equal(val[0, 0, which, h][one], x[2 * n, which, h])
            same[0, 0, which, h][one] = False
    assert np.array_equal(c.bits()[same], before[same])
