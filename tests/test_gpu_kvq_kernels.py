"""Attention over the 8-bit cache by each of its two kernels on the same batches (which one runs follows from the number of units and the width of the block
table: a slot of its own makes the table wide), and pages whose ids are bad for some rows of a sequence only."""
import numpy as np
import pytest
import torch

from paper_2605_08862_amd import binding as B
from paper_2605_08862_amd.runtime import KvqCache
from tests.test_gpu_kvq import DEV, Both, _close_on_gpu, _i32

pytestmark = pytest.mark.gpu

# Hq, Hkv, D, contexts, rows, tokens of a slot besides that makes the kernel for many rows run (tests/test_kvq_shares.py checks that it does, and without it not)
CASES = [
    (28, 4, 128, [700, 64, 1300, 0, 33, 129, 2000, 5, 640], [17, 16, 9, 1, 10, 4, 17, 13, 5], 40000),
    (28, 4, 64, [700, 64, 1300, 0, 33, 129, 2000, 5, 640], [17, 16, 9, 1, 10, 4, 17, 13, 5], 40000),
    (16, 2, 64, [500, 90, 0, 77, 1000, 31, 60] * 3, [7, 6, 3, 0, 1, 5, 7] * 3, 40000),            # two query tiles at most
    (16, 2, 128, [500, 90, 0, 77, 1000, 31, 60] * 3, [7, 6, 3, 0, 1, 5, 7] * 3, 40000),
    (8, 8, 64, [200, 63, 64, 1, 900], [40, 33, 64, 128, 1], 40000),                              # one query head to a KV head
    (128, 1, 128, [70, 0, 64, 300] * 5, [1, 3, 2, 1] * 5, 40000),                                # 128 to one
    (12, 2, 64, [0, 1000, 317], [400, 200, 1], 10000),                                           # pieces of prompts
]
IDS = ["q%d_kv%d_d%d_b%d_t%d_n%d" % (c[0], c[1], c[2], len(c[3]), max(c[3]), max(c[4])) for c in CASES]


def _filled_in(Hq, Hkv, D, ctx, counts, seed, besides):
    rng = np.random.default_rng(seed)
    n = len(ctx)
    slots = [int(s) for s in rng.permutation(n)]
    caps = [0] * n
    for b in range(n):
        caps[slots[b]] = max(ctx[b] + counts[b], 1)
    cache = KvqCache(1, Hq, Hkv, D, n + 1, 0, max(counts), device=DEV, page_perm_seed=seed, slot_tokens=caps + [max(besides, 1)])
    x = Both.__new__(Both)
    x.dims, x.caps, x.cache = (Hq, Hkv, D), caps, cache
    held = [c + r for c, r in zip(ctx, counts)]
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows = lambda size: torch.randn(sum(held), Hkv, D, generator=g, device=DEV).mul_(size).to(torch.bfloat16)
    k = rows(1.0)
    k[:, :, 5] *= 8.0
    cache.write(0, _i32(slots), _i32([0] * n), _i32(held), max(held), k, rows(0.7))
    return x, slots, torch.randn(sum(counts), Hq, D, generator=g, device=DEV).to(torch.bfloat16)


@pytest.mark.parametrize("wide", [False, True], ids=["few", "many"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_each_kernel_matches_the_oracle(case, wide):
    Hq, Hkv, D, ctx, counts, besides = case
    x, slots, q = _filled_in(Hq, Hkv, D, ctx, counts, len(ctx) + D, besides if wide else 0)
    M = sum(counts)
    out = torch.full((M + 2, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    args = (_i32(slots), _i32(ctx), _i32(counts), max(counts))
    x.cache.attention(0, q, *args, out=out)
    _close_on_gpu(x, out, q, slots, ctx, counts)
    first = out.clone()
    x.cache.attention(0, (q.float().flip(0) * -3.0).to(torch.bfloat16), *args, out=out)
    x.cache.attention(0, q, *args, out=out)
    assert torch.equal(out, first) and bool((out[M:] == 7.0).all()) and x.cache.poll_status() == 0


@pytest.mark.parametrize("Hq,Hkv,D,ctx,counts,page,besides", [
    (28, 4, 128, [30, 100], [9, 300], 5, 0),                               # rows 0 .. 219 of a piece of a prompt do not see its page 5
    (28, 4, 128, [30, 100], [9, 300], 5, 40000),
    (28, 4, 64, [30, 100], [9, 300], 1, 40000),                            # a page that every row sees
    (12, 2, 128, [9000, 70], [1, 17], 1, 0),                               # every row of a verify block sees it
    (12, 2, 128, [9000, 120], [1, 17], 2, 0),                              # rows 8 .. 16 of one block see page 2
    (28, 4, 128, [9000, 9020], [1, 17], 141, 0),                           # a unit cut into parts: rows 4 .. 16
    (28, 4, 128, [60] * 40 + [10000], [9] * 40 + [300], 160, 0),           # the same in the kernel for many rows
], ids=str)
def test_rows_beside_a_bad_page(Hq, Hkv, D, ctx, counts, page, besides):
    """Rows that see the page stay as they are; of those before them, and of the other sequences, what is written is right."""
    x, slots, q = _filled_in(Hq, Hkv, D, ctx, counts, 3, besides)
    args = (_i32(slots), _i32(ctx), _i32(counts), max(counts))
    b, clean = len(ctx) - 1, x.cache.attention(0, q, *args)
    seen = max(0, min(counts[b], page * 64 - ctx[b]))                      # rows below the page
    table, kept = x.cache.block_table, int(x.cache.block_table[slots[b], page])
    for bad in (-1, x.cache.n_pages):
        out = torch.full_like(q, 3.0)
        table[slots[b], page] = bad
        x.cache.attention(0, q, *args, out=out)
        assert x.cache.poll_status() == (B.BS_FAULT_KV_PAGES if seen < counts[b] else 0)
        table[slots[b], page] = kept
        first = sum(counts[:b])
        assert bool((out[first + seen:] == 3.0).all())
        left = (out == 3.0).all(-1, keepdim=True)
        assert not bool(left[:first].any())
        _close_on_gpu(x, torch.where(left, clean, out), q, slots, ctx, counts[:b] + [seen])


@pytest.mark.parametrize("wide", [False, True], ids=["few", "many"])
@pytest.mark.parametrize("k_size,v_size", [(2.0 ** -19, 2.0 ** -20), (1.0, 2.0 ** -17), (4000.0, 9000.0), (2.0 ** -6, 3.0)])
def test_smallest_and_largest_scales(k_size, v_size, wide):
    """Values that are subnormal in float16 (multiples of 2^-24), and scores of many thousands."""
    Hq, Hkv, D, ctx, counts = 28, 4, 128, [100, 0, 64, 257, 31, 5, 90, 200, 12], [9, 3, 1, 9, 2, 9, 9, 9, 9]
    rng = np.random.default_rng(17)
    held = [c + r for c, r in zip(ctx, counts)]
    n = len(ctx)
    cache = KvqCache(1, Hq, Hkv, D, n + 1, 0, max(counts), device=DEV, slot_tokens=held + [40000 if wide else 1])
    x = Both.__new__(Both)
    x.dims, x.caps, x.cache = (Hq, Hkv, D), held, cache
    k, v = (torch.from_numpy(rng.normal(0, s, (sum(held), Hkv, D))).to(torch.bfloat16).to(DEV) for s in (k_size, v_size))
    slots = list(range(n))
    cache.write(0, _i32(slots), _i32([0] * n), _i32(held), max(held), k, v)
    q = torch.from_numpy(rng.normal(0, 1.0, (sum(counts), Hq, D))).to(torch.bfloat16).to(DEV)
    out = cache.attention(0, q, _i32(slots), _i32(ctx), _i32(counts), max(counts))
    _close_on_gpu(x, out, q, slots, ctx, counts)
    assert cache.poll_status() == 0
