"""Attention over the 8-bit cache where units are cut into so many parts that one of them has no neighbour on a level of the merge: against the oracle in
float64, on a workspace that holds nothing yet and on one that holds the partial results of another batch."""
import pytest
import torch

from tests.test_gpu_kvq import DEV, _close_on_gpu, _filled, _i32

pytestmark = pytest.mark.gpu

# Hq, Hkv, D, contexts, rows, {(parts fold in eights, level without a neighbour)} that the case is for (tests/test_kvq_shares.py checks that it reaches them)
CASES = [
    (12, 2, 128, [4250], [1], {(True, 0)}),
    (12, 2, 128, [17000], [1], {(True, 0)}),
    (12, 2, 128, [34000], [1], {(True, 1)}),
    (12, 2, 128, [36000], [1], {(True, 1)}),
    (12, 2, 128, [2250], [9], {(False, 0)}),
    (12, 2, 128, [4900], [22], {(False, 0)}),
    (28, 4, 128, [9000], [17], {(False, 0), (False, 1)}),
    (28, 4, 128, [10000], [17], {(False, 1)}),
    (28, 4, 128, [9000] * 3, [1] * 3, {(True, 0)}),
    (8, 2, 64, [4300], [1], {(True, 0)}),
    (28, 4, 128, [10000] + [60] * 40, [17] + [9] * 40, {(False, 1)}),         # the kernel for many rows
    (28, 4, 128, [26000] + [60] * 40, [17] + [9] * 40, {(False, 0), (False, 1)}),
    (28, 4, 64, [12000] + [60] * 40, [17] + [9] * 40, {(False, 0)}),
]
IDS = ["q%d_kv%d_d%d_b%d_t%d_n%d" % (c[0], c[1], c[2], len(c[3]), max(c[3]), max(c[4])) for c in CASES]


@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_units_with_a_lone_part(case):
    Hq, Hkv, D, ctx, counts, _ = case
    x, slots, q = _filled(Hq, Hkv, D, ctx, counts, seed=sum(ctx) + D)
    args = (_i32(slots), _i32(ctx), _i32(counts), max(counts))
    other = (q.float().flip(0) * -3.0).to(torch.bfloat16)                    # other maxima and sums in the same places
    first = x.cache.attention(0, q, *args)
    _close_on_gpu(x, first, q, slots, ctx, counts)
    for _ in range(3):
        x.cache.attention(0, other, *args)
        again = x.cache.attention(0, q, *args)
        assert torch.equal(again, first)
    short = [max(c // 3, 1) for c in ctx]                                    # another cut of the same slots
    x.cache.attention(0, other, args[0], _i32(short), *args[2:])
    assert torch.equal(x.cache.attention(0, q, *args), first) and x.cache.poll_status() == 0
