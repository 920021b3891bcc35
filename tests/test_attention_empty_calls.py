"""Calls with nothing to do, on the CPU: the address of an empty tensor is NULL, and such calls are taken."""
import torch

import paper_2411_15715_amd as si
from test_attention_host import BASE, append, attend, cache, norm, refused

NULL = torch.empty((0, 64)).data_ptr() or None


def test_no_rows():
    si.si_norm(norm(rows=0, r=NULL, y=NULL, gate=NULL, out=NULL, r_out=NULL))
    si.si_norm(norm(rows=0, r=NULL, y=NULL, out=NULL, r_out=NULL, post=si.SI_NORM_RMS, w_post=BASE))
    for kw in (dict(d=0), dict(eps=-1.0), dict(pre=7)):
        refused(si.si_norm, norm(rows=0, **kw))


def test_no_tokens():
    si.si_cache_append(cache(), 0, append(n_tokens=0, q=NULL, k=NULL, v=NULL, q_out=NULL, seq=NULL, pos=NULL))
    si.si_cache_append(cache(), 1, append(n_tokens=0, k=NULL, v=NULL, q_out=NULL, seq=NULL, pos=NULL))
    refused(si.si_cache_append, cache(), 2, append(n_tokens=0))
    refused(si.si_cache_append, cache(type=7), 0, append(n_tokens=0))


def test_no_sequences():
    si.si_attend(cache(), 0, attend(n=0, q=NULL, out=NULL, lse=NULL, seqs=NULL))
    si.si_attend(cache(max_pages=1000), 0, attend(n=0, q=NULL, out=NULL, max_len=50000, scratch=None))
    refused(si.si_attend, cache(), 2, attend(n=0))
    refused(si.si_attend, cache(), 0, attend(n=0, n_new=0))
