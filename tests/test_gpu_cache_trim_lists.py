"""si_cache_trim with sequences that a list names more than once: taken in list order, tables and status alike, whichever block runs first."""
import random

import pytest

import paper_2411_15715_amd as si
from test_gpu_cache_pages import Pool, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep,status", [([5, 3], 0), ([3, 5], si.SI_CACHE_BAD_LEN), ([4, 4], 0), ([-1, 3], si.SI_CACHE_BAD_LEN), ([99, 70], si.SI_CACHE_BAD_LEN),
                                         ([70, 33], 0), (None, 0), ([64, 0], 0), ([0, 1], si.SI_CACHE_BAD_LEN), ([80, 80], 0)])
def test_a_sequence_named_twice(keep, status):
    for _ in range(5):
        p = Pool()
        p.extend([1, 2, 3], [40, 80, 9])
        want = p.books.trim([2, 2], keep)
        assert want == status
        two, k = dev([2, 2]), dev(keep) if keep is not None else None
        si.si_cache_trim(p.c.desc, two.data_ptr(), 2, k.data_ptr() if k is not None else None, p.stream)
        p.check(want)
        p.extend([2], [50])


def test_shared_pages_and_lists_that_name_a_sequence_often():
    """Entries of a sequence further apart than a wave is wide, between those of others that share its pages."""
    r = random.Random(3)
    p = Pool(n_pages=200, n_seqs=40, max_pages=6)
    p.extend(list(range(20)), [32 * 5 + 7] * 20)
    p.fork([0, 1, 2, 3, 3, 3], [30, 31, 32, 33, 34, 35])
    for rounds in range(3):
        lens = [int(x) for x in p.books.lens]
        seqs = [r.choice([0, 1, 2, 3, 30, 33, 34, 35, 19, 99, -1, r.randrange(20)]) for _ in range(si.SI_CACHE_MAX_LIST)]
        p.trim(seqs, [r.randint(max(0, lens[s] - 60 * i // len(seqs) - 5), lens[s]) if 0 <= s < 40 else r.randint(-1, 3) for i, s in enumerate(seqs)])
    p.trim([3, 33, 3, 34, 33], [40, 33, 1, 64, 0])
