"""Pages that a sequence names and whose count says that they are free: extending and forking report them and change nothing, as the page would be
given to somebody else beside its owner."""
import pytest
import torch

import paper_2411_15715_amd as si
from test_gpu_cache_pages import Pool, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [0, -1, -0x80000000])
@pytest.mark.parametrize("entry", [0, 1, 2])
def test_a_page_in_use_with_no_count(entry, count):
    p = Pool()
    p.extend([0, 1], [40, 32 * 2 + 5])
    page = int(p.c.table[1, entry])
    a, b = dev([1]), dev([3])
    seq, pos = dev([7, 7]), dev([7, 7])
    p.c.refs[page] = count
    si.si_cache_fork(p.c.desc, a.data_ptr(), b.data_ptr(), 1, p.stream)
    torch.cuda.synchronize()
    assert int(p.c.status.item()) == si.SI_CACHE_BAD_PAGE and int(p.c.refs[page]) == count
    p.c.status.zero_()
    if entry == 2:  # the partly filled one
        si.si_cache_extend(p.c.desc, a.data_ptr(), 1, None, 2, seq.data_ptr(), pos.data_ptr(), 2, p.stream)
        torch.cuda.synchronize()
        assert int(p.c.status.item()) == si.SI_CACHE_BAD_PAGE and int(p.c.refs[page]) == count and seq.tolist() == [-1, -1]
        p.c.status.zero_()
    p.c.refs[page] = 1
    p.check()
    p.fork([1], [3])
    p.extend([1, 3], [40, 1])
