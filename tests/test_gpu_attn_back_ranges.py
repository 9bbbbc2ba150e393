"""Gradients of windowed attention in fp16 where rows, heads and sequences are of very different sizes.

Every product and sum of a row's gradient is linear in its dout, so dout times a power of two is the gradient times that power, to the last bit, as long as
neither leaves the type's normal range: a row's bits do not depend on what else is in the call.  The same holds for a key and all rows that see it.
Values in keys that nothing sees change nothing."""
import pytest
import torch

import attention_back_ref as R
from test_gpu_attn_back import ALL, call, compare, make, starts

pytestmark = pytest.mark.gpu
F16 = torch.float16

# rows see few keys (weights as two values) and many, walks that are split, first tokens' rows that go to workgroups of their own, every width of head
CASES = [
    ([(300, 300), (40, 170), (1, 33)], 4, 2, 64, 50, 0, 3),
    ([(700, 700), (300, 300)], 2, 1, 128, 600, 0, 0),
    ([(600, 1500)], 4, 2, 128, ALL, 0, 0),
    ([(700, 700)], 2, 2, 32, 20, 0, 5),
    ([(4, 2500), (3, 700)], 4, 1, 128, ALL, 0, 0),
    ([(2000, 40)], 4, 1, 80, ALL, ALL, 0),
    ([(900, 900)], 2, 1, 24, 700, 10, 40),
]


def factor(power):
    """2^power to the last bit (a GPU's power function need not be that exact)."""
    return torch.tensor([2.0 ** -i for i in range(13)], dtype=torch.float64, device=power.device)[-power.long()]


def scaled(x, power):
    return (x.double() * factor(power)).to(F16)


def same(small, large, power, what):
    """small = large * 2^power to the last bit, wherever that is a normal number."""
    exp = large.double() * factor(power)
    there = exp.abs() >= 2.0 ** -14
    assert there.sum() > exp.numel() // 50, what
    off = (small.double() != exp) & there
    assert not off.any(), (what, int(off.sum()), int(there.sum()))


def large_dout(case, seed):
    """Tensors whose dout has no number that 2^-12 would take out of the normal range, and whose gradients are large."""
    lens, Hq, Hk, D, left, right, sinks = CASES[case]
    (q, k, v, dout), where = make(lens, Hq, Hk, D, F16, seed)
    q.mul_(2.0)
    dout.mul_(2.0 ** 9)
    dout[dout.abs() < 0.25] = 0.25
    return lens, (q, k, v, dout), where, (left, right, sinks)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_of_different_sizes(case):
    """Each row and head of the queries by a power of its own, down to 2^-12: dq follows to the last bit."""
    lens, (q, k, v, dout), where, window = large_dout(case, 40 + case)
    _, _, (dq, _, _) = call((q, k, v, dout), where, *window)
    g = torch.Generator().manual_seed(case)
    power = -torch.randint(0, 13, (q.shape[0], q.shape[1], 1), generator=g).cuda()
    _, _, (mine, _, _) = call((q, k, v, scaled(dout, power)), where, *window)
    same(mine, dq, power, "dq")


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("by", ["sequences", "key heads"])
def test_sequences_and_heads_of_different_sizes(case, by):
    """All rows that see a key by one power: dk and dv follow to the last bit."""
    lens, (q, k, v, dout), where, window = large_dout(case, 50 + case)
    Hq, Hk = q.shape[1], k.shape[1]
    _, _, plain = call((q, k, v, dout), where, *window)
    pq, pk = torch.zeros(q.shape[0], Hq, 1).cuda(), torch.zeros(k.shape[0], Hk, 1).cuda()
    if by == "sequences":
        cq, ck = starts([a for a, _ in lens]), starts([b for _, b in lens])
        for s in range(len(lens)):
            pq[cq[s]:cq[s + 1]] = pk[ck[s]:ck[s + 1]] = -12 if s % 2 == 0 else 0
    else:
        for h in range(Hk):
            pk[:, h] = -12 if h % 2 == 0 else 0
            pq[:, h * Hq // Hk:(h + 1) * Hq // Hk] = -12 if h % 2 == 0 else 0
    _, _, got = call((q, k, v, scaled(dout, pq)), where, *window)
    for name, y, x, p in zip(("dq", "dk", "dv"), got, plain, (pq, pk, pk)):
        same(y, x, p, name)


def test_keys_that_only_small_rows_see():
    """The last rows of a window of 50 by 2^-12: the keys that no other row sees follow."""
    lens, Hq, Hk, D, window = [(400, 400)], 2, 1, 64, (50, 0, 0)
    (q, k, v, dout), where = make(lens, Hq, Hk, D, F16, 60)
    dout.mul_(2.0 ** 9)
    dout[dout.abs() < 0.25] = 0.25
    _, _, plain = call((q, k, v, dout), where, *window)
    power = torch.zeros(400, 1, 1).cuda()
    power[200:] = -12
    _, _, got = call((q, k, v, scaled(dout, power)), where, *window)
    same(got[0], plain[0], power, "dq")
    for n in (1, 2):
        same(got[n][200:], plain[n][200:], power[200:], "keys")
        assert torch.equal(got[n][:150], plain[n][:150])


@pytest.mark.parametrize("case", [0, 1, 2, 3, 4, 6])
def test_values_of_keys_that_nobody_sees(case):
    """Keys before the first row's window, with the largest values of the type: nothing changes, and their own gradients stay zero."""
    lens, Hq, Hk, D, left, _, _ = CASES[case]
    lens, left = [(a, b + 40) for a, b in lens], min(left, 30)
    tensors, where = make(lens, Hq, Hk, D, F16, 70 + case)
    _, _, plain = call(tensors, where, left, 0, 0)
    ck = starts([b for _, b in lens])
    unseen = []
    for s, (a, b) in enumerate(lens):
        see = R.seen(a, b, left, 0, 0).any(0)
        unseen += [ck[s] + int(j) for j in (~see).nonzero()[:, 0]]
    assert unseen
    q, k, v, dout = tensors
    v[unseen] = 65504.0
    _, _, got = call((q, k, v, dout), where, left, 0, 0)
    assert all(torch.equal(a, b) for a, b in zip(got, plain))


@pytest.mark.parametrize("case", range(len(CASES)))
def test_large_values_that_few_rows_see(case):
    """One key's values 2^10 times the others': rows that do not see it are as they were, those that do are right."""
    lens, Hq, Hk, D, left, right, sinks = CASES[case]
    tensors, where = make(lens, Hq, Hk, D, F16, 80 + case)
    _, _, plain = call(tensors, where, left, right, sinks)
    a, b = lens[0]
    token = b - 1
    q, k, v, dout = tensors
    v[token] *= 2.0 ** 10
    _, _, got = call((q, k, v, dout), where, left, right, sinks)
    see = R.seen(a, b, left, right, sinks)[:, token]
    assert torch.equal(got[0][:a][~see.cuda()], plain[0][:a][~see.cuda()])
    compare(lens, (q, k, v, dout), left, right, sinks, got)


def test_against_the_definition():
    """Sequences 2^12 apart, each within the bound of its own sizes."""
    lens, Hq, Hk, D, left, right, sinks = CASES[0]
    (q, k, v, dout), where = make(lens, Hq, Hk, D, F16, 90)
    dout[:lens[0][0]] *= 2.0 ** -6
    dout[lens[0][0]:] *= 2.0 ** 8
    _, _, got = call((q, k, v, dout), where, left, right, sinks)
    compare(lens, (q, k, v, dout), left, right, sinks, got)
