"""si_attend_shared on the stand-in for the HIP runtime: calls that need no scratch are taken without one, and what is launched."""
import pytest

from test_host_calls import host  # noqa: F401

SETUP = """
buf = np.zeros(1 << 16, np.uint8)
base = (buf.ctypes.data + 255) // 256 * 256
cache = lambda kind=si.SI_KV_BF16, d=128, kv=8: si.si_cache_t(pages=base, table=base, lens=base, refs=base, status=base, n_pages=4, page_tokens=64, n_layers=2, n_kv_heads=kv, head_dim=d, type=kind, n_seqs=4,
                                                              max_pages=2000)

def attend(d=128, heads=32, **kw):
    o = dict(q=base, out=base, lse=base, seqs=base, q_stride=heads * d, out_stride=heads * d, n=1, n_new=1, n_heads=heads, max_len=200)
    o.update(kw)
    return si.si_attend_t(**o)

def launched(c, a):
    log()
    rc = attempt(si.si_attend_shared, c, 0, a)
    return rc, [l.split()[0] for l in log() if l.startswith("k_")]
"""


@pytest.mark.parametrize("call", ["n=1, max_len=200", "n=1, max_len=0", "n=1, max_len=1", "n=1, n_new=3, max_len=64", "n=1, max_len=200, window=50"])
def test_calls_that_need_no_scratch_are_taken_without_one(host, call):  # noqa: F811
    host(SETUP + """
for kind, d in ((si.SI_KV_BF16, 128), (si.SI_KV_BF16, 64), (si.SI_KV_E4M3, 192)):
    c, a = cache(kind, d), attend(d, %s)
    assert si.si_attend_scratch_bytes(c, a) == si.si_attend_shared_scratch_bytes(c, a) == 0
    assert launched(c, a) == (si.SI_OK, ["k_attend"])
    a.scratch, a.scratch_bytes = base + 4, 0  # (not looked at)
    assert launched(c, a) == (si.SI_OK, ["k_attend"])
""" % call)


def test_calls_that_need_scratch_are_refused_without_it(host):  # noqa: F811
    host(SETUP + """
for a in (attend(n=1, max_len=100000), attend(n=2, max_len=200), attend(n=4, max_len=100000)):
    c = cache()
    need = si.si_attend_shared_scratch_bytes(c, a)
    assert need > 0
    for scratch, n in ((None, need), (None, 0), (base, need - 1), (base, 0), (base + 8, need)):
        a.scratch, a.scratch_bytes = scratch, n
        assert launched(c, a) == (si.SI_EINVAL, [])
    a.scratch, a.scratch_bytes = base, need
    assert launched(c, a)[0] == si.SI_OK
a = attend(n=4, max_len=100000, scratch=base, scratch_bytes=1 << 40)
assert launched(cache(), a) == (si.SI_OK, ["k_share", "k_attend_pieces", "k_join_pieces"])
""")
