"""si_attend with more rows than a launch could hold joining blocks for: a block for each sequence, whatever max_len says.  Against torch in 64 bits, with the
tolerances of test_gpu_attend.py but for the weights (2^-16 of each)."""
import numpy as np
import pytest
import torch

import paper_2411_15715_amd as si
from attention_reference import Cache

pytestmark = pytest.mark.gpu


def test_many_sequences_of_many_rows():
    n, n_new, kv, per, d, page = 1024, 8, 128, 16, 64, 32
    c = Cache(si.SI_KV_BF16, 4, page, n, 160, 1, kv, d, seed=2)
    c.table[:, 0] = torch.arange(n, dtype=torch.int32) % 4
    lens = 8 + torch.arange(n, dtype=torch.int32) % 25
    c.lens.copy_(lens)
    row = kv * per * d
    q = torch.randn((n * n_new, row), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(torch.bfloat16)
    out, lse = torch.full_like(q, 99.0), torch.full((n * n_new, kv * per), 99.0, device="cuda")
    desc = si.si_attend_t(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), q_stride=row, out_stride=row, n=n, n_new=n_new, n_heads=kv * per, max_len=5000)
    desc.scratch_bytes = si.si_attend_scratch_bytes(c.desc, desc)
    scratch = torch.zeros(desc.scratch_bytes, dtype=torch.uint8, device="cuda")
    desc.scratch = scratch.data_ptr()
    print("attend", dict(n=n, rows=n_new * per, kv=kv, scratch=desc.scratch_bytes), flush=True)
    si.si_attend(c.desc, 0, desc, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    for s in (0, 1, 511, 1022, 1023):
        L = int(lens[s])
        k, v = (torch.from_numpy(a).cuda() for a in c.gather(0, s, L))
        qq = q[s * n_new:(s + 1) * n_new].double().view(n_new, kv, per, d).transpose(0, 1)  # [kv][n_new][per][d]
        x = qq.reshape(kv, n_new * per, d) @ k.transpose(1, 2).contiguous() * d ** -0.5
        see = torch.arange(L, device="cuda") < (L - n_new + 1 + torch.arange(n_new, device="cuda").repeat_interleave(per))[:, None]
        x = x.masked_fill(~see, -np.inf)
        p = x.softmax(-1)
        o, mag = p @ v, p @ v.abs()
        mag_s = (qq.reshape(kv, n_new * per, d).abs() @ k.abs().transpose(1, 2).contiguous() * d ** -0.5).amax(-1, keepdim=True)
        ds, sums = (d * 2.0 ** -23 + 2.0 ** -22) * mag_s, (L / 16 + 64) * 2.0 ** -23
        want = x.logsumexp(-1)
        shape = lambda t: t.double().view(n_new, kv, per, -1).transpose(0, 1).reshape(kv, n_new * per, -1)  # noqa: E731
        got, got_lse = shape(out[s * n_new:(s + 1) * n_new]), shape(lse[s * n_new:(s + 1) * n_new])[..., 0]
        assert bool(((got_lse - want).abs() <= ds[..., 0] + sums + 2.0 ** -22 * want.abs()).all())
        assert bool(((got - o).abs() <= 2.0 ** -8 * o.abs() + 1.01 * (2.0 ** -16 + 2 * ds + 2 * sums) * mag).all())
