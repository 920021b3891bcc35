"""si_sample on the CPU: what it refuses before any GPU call, and the size of its scratch."""
import ctypes

import numpy as np
import pytest

import paper_2411_15715_amd as si

BUF = np.zeros(1 << 12, np.uint8)
BASE = (BUF.ctypes.data + 255) // 256 * 256


def desc(**kw):
    d = dict(logits=BASE, temperature=BASE, top_k=BASE, top_p=BASE, min_p=BASE, u=BASE, token=BASE, prob=BASE, kept=BASE, scratch=BASE, scratch_bytes=1 << 40, stride=1000, rows=3,
             vocab=1000, type=si.SI_F32)
    d.update(kw)
    return si.si_sample_t(**d)


def refused(f, *args):
    with pytest.raises(si.ScheInferError) as e:
        f(*args)
    assert e.value.code == si.SI_EINVAL and "si_sample" in str(e.value)


@pytest.mark.parametrize("kw", [dict(type=2), dict(type=-1), dict(rows=-1), dict(rows=si.SI_SAMPLE_MAX_ROWS + 1), dict(vocab=0), dict(vocab=-5), dict(vocab=si.SI_SAMPLE_MAX_VOCAB + 1, stride=1 << 30),
                                dict(rows=65536, vocab=1 << 20, stride=1 << 20)])
def test_bad_shapes_are_refused(kw):
    refused(si.si_sample, desc(**kw))
    refused(si.si_sample_scratch_bytes, desc(**kw))


@pytest.mark.parametrize("kw", [dict(logits=None), dict(u=None), dict(token=None), dict(scratch=None), dict(logits=BASE + 2), dict(logits=BASE + 1, type=si.SI_BF16), dict(temperature=BASE + 2),
                                dict(top_k=BASE + 1), dict(top_p=BASE + 2), dict(min_p=BASE + 3), dict(u=BASE + 2), dict(token=BASE + 2), dict(prob=BASE + 2), dict(kept=BASE + 2),
                                dict(scratch=BASE + 8), dict(stride=999), dict(stride=-1000), dict(scratch_bytes=1 << 10)])
def test_bad_pointers_strides_and_scratch_are_refused(kw):
    refused(si.si_sample, desc(**kw))


def test_missing_descriptors_are_refused():
    assert si.lib().si_sample(None, None) == si.SI_EINVAL
    assert si.lib().si_sample_scratch_bytes(None) == si.SI_EINVAL


def test_no_rows_is_a_no_op():
    si.si_sample(si.si_sample_t(rows=0, vocab=10))


def test_scratch_serves_smaller_calls():
    most = si.si_sample_scratch_bytes(desc(rows=40, vocab=70000))
    assert most % 16 == 0
    for rows in (0, 1, 17, 40):
        for vocab in (1, 8192, 8193, 70000):
            assert si.si_sample_scratch_bytes(desc(rows=rows, vocab=vocab)) <= most
