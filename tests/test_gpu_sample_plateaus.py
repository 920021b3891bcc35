"""si_sample on rows with a few heavy plateaus of equal logits, where top_p ends at a plateau's end or a little beyond it: more tokens of one value than are put in
order at once, and sums whose parts differ by 2^20 and more.

The expected number of tokens is formed with sums of 64-bit mantissas of the weights as the header has them, multiples of 2^-(62 - ceil(log2 vocab)), up to
top_p times the sum of the weights as they are.  Every p of the tests is 1e-11 of the sum or more away from the border between two numbers of tokens
(checked here, on the CPU): sums of doubles are some 1e-14 off, a weight next to a multiple may be cut to the one below, those here 2^-64 times 131072."""
import numpy as np
import pytest
import torch

from test_gpu_sample import sample

pytestmark = pytest.mark.gpu


def expected(l, t, p):
    """number of tokens left, indices left, their weights; None where p is too near to a border"""
    w = np.exp((l.astype(np.float64) - float(l.max())) / t).astype(np.longdouble)
    goal = np.longdouble(p) * np.sum(w)
    unit = np.longdouble(2.0) ** (int(np.ceil(np.log2(len(l)))) - 62)
    w = np.floor(w / unit) * unit
    order = np.argsort(-l, kind="stable")
    sums = np.cumsum(w[order])
    n = 1 + int(np.searchsorted(sums, goal))
    if sums[n - 1] - goal < 1e-11 * sums[-1] or goal - (sums[n - 2] if n > 1 else 0) < 1e-11 * sums[-1]:
        return None
    left = np.sort(order[:n])
    return n, left, w[left]


def check_rows(l, t, ps, dtype=torch.float32, seed=0):
    """l: numpy fp32 [vocab], each p a row of its own; tokens drawn with numbers away from borders"""
    rng = np.random.default_rng(seed)
    t = float(np.float32(t))
    rows = [(p, e) for p, e in ((float(np.float32(p)), expected(l, t, float(np.float32(p)))) for p in ps) if e is not None]
    assert len(rows) >= min(2, len(ps))
    us, tokens, probs = [], [], []
    for _, (n, left, w) in rows:
        sums = np.cumsum(w)
        while True:
            u = float(rng.random(dtype=np.float32))
            at = int(np.searchsorted(sums, u * sums[-1], side="right"))
            if abs(u * sums[-1] - sums[at]) > 1e-7 * sums[-1] and (at == 0 or abs(u * sums[-1] - sums[at - 1]) > 1e-7 * sums[-1]):
                break
        us.append(u)
        tokens.append(int(left[at]))
        probs.append(float(w[at] / sums[-1]))
    x = torch.from_numpy(l).to("cuda", dtype)
    assert np.array_equal(x.float().cpu().numpy(), l)
    print("plateaus", len(l), dtype, [p for p, _ in rows], flush=True)
    token, prob, kept = sample(x[None].expand(len(rows), len(l)), dict(temperature=[t] * len(rows), top_p=[p for p, _ in rows]), us, stride=0)
    assert kept.tolist() == [e[0] for _, e in rows]
    assert token.tolist() == tokens
    assert np.all(np.abs(prob - np.array(probs)) <= (2.0 ** -24 + 2.0 ** -25) * np.array(probs) + 2.0 ** -42)


def plateaus(vocab, parts, seed=0):
    """parts: (tokens, logit), the last for all that are left; in shuffled order"""
    l = np.full(vocab, parts[-1][1], np.float32)
    at = 0
    for n, v in parts[:-1]:
        l[at:at + n] = v
        at += n
    np.random.default_rng(seed).shuffle(l)
    return l


def around(l, t, n, steps):
    """fp32 values next to the share of the n largest tokens"""
    w = np.exp((l.astype(np.float64) - float(l.max())) / float(np.float32(t))).astype(np.longdouble)
    p = np.float32(np.sum(np.sort(w)[::-1][:n]) / np.sum(w))
    out = []
    for k in range(-steps, steps + 1):
        q = p
        for _ in range(abs(k)):
            q = np.nextafter(q, np.float32(2 if k > 0 else -1))
        out.append(float(q))
    return [q for q in out if q < 1]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("last", [-16.5, -5.59375])
@pytest.mark.parametrize("t", [1.0, 1.1, 1.3, 1.5])
def test_top_p_at_the_end_of_a_plateau(dtype, last, t):
    l = plateaus(131072, [(4000, 0.0), (56000, -2.296875), (0, last)])
    check_rows(l, t, around(l, t, 60000, 10), dtype)
    check_rows(l, t, around(l, t, 4000, 4), dtype)


def test_plateaus_that_are_not_multiples_of_anything():
    l = plateaus(131072, [(4000, 0.0), (56000, -2.3), (0, -16.6)])
    check_rows(l, 1.3, around(l, 1.3, 60000, 10))
    l = plateaus(100003, [(3000, 7.7), (2500, 7.1), (9000, 3.3), (30000, -4.4), (0, -9.9)], seed=1)
    for n in (5500, 14500, 44500):
        for t in (0.8, 0.9, 1.0):
            check_rows(l, t, around(l, t, n, 7))


def test_values_between_the_plateaus():
    rng = np.random.default_rng(3)
    l = plateaus(131072, [(5000, 0.0), (60000, -3.0), (0, -14.0)], seed=2)
    some = rng.choice(131072, 20000, replace=False)
    l[some] = rng.uniform(-15, -1, 20000).astype(np.float32)
    n = int(np.sum(l >= -3.0))
    check_rows(l, 1.1, around(l, 1.1, n, 10))
    check_rows(l, 1.1, [0.3, 0.5, 0.9, 0.99, 0.9999])
