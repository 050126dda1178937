"""The 8-bit session cache on the GPU where its calls are easiest to get wrong: sessions whose offsets contradict each
other, rows that one key dominates, the log-sum-exp's last bits, the ends of the number formats, what is not finite, and
work that is dealt out in equal shares."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu

ts = pytest.importorskip("paper_2606_19271_amd")

PAGE = 64


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ts.load_cache()
    return torch.device("cuda:0")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def filled(g, lens, H, d, k=1.0, v=1.0, spare=0):
    """A pool that holds sessions of these lengths, appended in one call, and their table."""
    need = [-(-n // PAGE) for n in lens]
    width = max(need + [1])
    order = torch.randperm(sum(need) + spare, generator=g, device="cuda").tolist()
    cache = ts.session_cache(max(1, sum(need) + spare), H, d)
    table = [[order.pop() for _ in range(n)] + [-1] * (width - n) for n in need]
    cu = [0] + np.cumsum(lens).tolist()
    k = (normal(g, cu[-1], H, d) * k).bfloat16() if not torch.is_tensor(k) else k
    v = (normal(g, cu[-1], H, d) * v).bfloat16() if not torch.is_tensor(v) else v
    ts.ts_cache_append(cache, k, v, ints(cu), max(lens + [1]), ints(table), ints([0] * len(lens)))
    return cache, table


def same(a, b):
    return all(torch.equal(x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32), y.view(
        torch.int16 if y.dtype == torch.bfloat16 else torch.int32)) for x, y in zip(a, b))


# ---- offsets that contradict each other

# (offsets, most rows): a backward session is skipped, and those after it name rows that earlier ones have
OVERLAPS = [([0, 1000, 0, 1000, 0, 1000, 2000], 1000), ([0, 1000, 0, 3000, 4000], 3000), ([0, 1000] * 35 + [2000], 1000)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 3])
@pytest.mark.parametrize("cu,most", OVERLAPS)
def test_attn_sessions_that_overlap_leave_the_others_alone(cu, most, splits, d):
    """More row tiles than disjoint sessions could have: the last session, the shortest and of rows that nobody else
    names, gets the result that it gets alone."""
    g = gen(len(cu) + splits + d)
    H, n = 12, len(cu) - 1
    lens = [200] * (n - 1) + [90]
    cache, table = filled(g, lens, H, d)
    q = normal(g, cu[-1], H, d).bfloat16()
    out, lse = torch.full_like(q, 7.0), torch.full((cu[-1], H), 7.0, device="cuda")
    ts.ts_cache_attn(q, cache, ints(cu), most, ints(table), ints(lens), 256, out=out, lse=lse, num_splits=splits)
    rows = slice(cu[-2], cu[-1])
    alone = ts.ts_cache_attn(q[rows].contiguous(), cache, ints([0, cu[-1] - cu[-2]]), most, ints(table[-1:]), ints(lens[-1:]), 256,
                             return_lse=True, num_splits=max(splits, 1))
    # two results, each off by a rounding of the weights and one of the result: 2^-8 of an average of the values' sizes each
    assert (out[rows].float() - alone[0].float()).abs().max() <= 4 * 2.0 ** -8 * 6
    assert (lse[rows] - alone[1]).abs().max() <= 1e-4
    assert torch.all(out[:cu[-2]] != 7.0)
