"""The attention over the paged cache where value scales are of very different size and where offsets reach past the call's rows.
All rows are held against the definition in 64 bits, on the GPU."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_verify import DEV, TYPES, Paged, half, i32, prefix

pytestmark = pytest.mark.gpu


def check(p, q, out, lse, scale, window=0, floor=0.0):
    """Rows and log-sums of every token of `q` against float64.  The limit: scores are dim products summed in float32 (2^-23 a step)
    and two more roundings; a probability is rounded to the type once, the exponential and the sums are float32; float16 has its
    fixed step below 2^-14.  `floor`: a step that a key adds besides, for each unit of its held value."""
    dtype, at, heads = q.dtype, 0, q.shape[1]
    group = heads // p.heads
    for b, m in enumerate(p.new):
        k, v, there = p.rows(b)
        rows = q[at:at + m].double()                             # fewer where the call has no more
        if len(rows) == 0:
            at += m
            continue
        k, v = (torch.from_numpy(np.ascontiguousarray(x)).to(DEV).repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))
        x = rows.transpose(0, 1)
        pos = torch.arange(len(rows), device=DEV)[:, None] + p.length[b] - m
        j = torch.arange(p.length[b], device=DEV)[None]
        see = (j <= pos) & torch.from_numpy(there).to(DEV)
        if window:
            see &= j > pos - window
        if p.length[b] == 0:
            want, log = torch.zeros_like(x), torch.full(x.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
            size, reach, most = want, torch.zeros_like(log), 0.0
        else:
            s = (x @ k.transpose(1, 2) * scale).masked_fill(~see, -math.inf)
            top = s.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            e = torch.exp(s - top)
            total = e.sum(-1, keepdim=True)
            log = (top + total.log())[..., 0]
            prob = e / total.clamp_min(1e-300)
            want, size, most = prob @ v, prob @ v.abs(), v.abs().max()
            reach = (abs(scale) * (x.abs() @ k.abs().transpose(1, 2))).masked_fill(~see, 0.0).amax(-1)
        keys = max(p.length[b], 1)
        ds = (p.dim + 4) * 2.0 ** -23 * reach
        limit = size * (half(dtype) * 1.01 + 2 * ds[..., None] + (keys + 64) * 2.0 ** -23) + half(dtype) * want.abs() * 1.01 + floor * keys
        limit = limit + 2.0 ** -25 * (dtype == torch.float16) * (1 + keys * most)
        got = out[at:at + len(rows)].double().transpose(0, 1)
        bad = ((got - want).abs() > limit) | got.isnan()
        assert not bad.any(), (b, int(bad.sum()), float(((got - want).abs() / limit.clamp_min(1e-300)).nan_to_num(math.inf).max()))
        if lse is not None:
            got = lse[at:at + len(rows)].double().transpose(0, 1)
            none = ~see.any(-1) if p.length[b] else torch.ones_like(pos[:, 0], dtype=torch.bool)
            assert (got[:, none] == -math.inf).all()
            off = (got - log).abs() - (ds + (keys + 64) * 2.0 ** -23 + 2.0 ** -22 * log.abs())
            assert (off[:, ~none] <= 0).all(), (b, float(off[:, ~none].max()))
        at += m


def attend(p, dtype, q_heads, window=0, scale=None, seed=5, floor=0.0, **kw):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randn(sum(p.new), q_heads, p.dim, generator=g, device=DEV).to(dtype)
    out, lse = p.cache.attend(q, *p.tokens(), scale=scale, window=window, lse=True, **kw)
    check(p, q, out, lse, p.dim ** -0.5 if scale is None else scale, window, floor)
    return q, out, lse


# ---- value scales -------------------------------------------------------------------------------------------------------

def value_scale(p, b, first, last, by, keep):
    """Value scales of positions first .. last - 1 of request b: times `by`, or `by` itself."""
    for t in range(first, last):
        spot = p.cache.v_scale[int(p.table[b][t // p.page]), :, t % p.page]
        spot.copy_(spot * by if keep else torch.full_like(spot, by))


@pytest.mark.parametrize("store,dtype", [("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("low", [0.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -100, 2.0 ** -60])
@pytest.mark.parametrize("high", [1.0, 2.0 ** 20, 2.0 ** 100])
@pytest.mark.parametrize("dim,group,new", [(64, 1, [1, 1, 1]), (128, 4, [3, 1, 70])])
def test_rows_of_zeros_and_of_large_values_in_one_cache(store, dtype, low, high, dim, group, new):
    # whole units of keys with the least scales there are, before, after and without ordinary ones: they count in the sums
    if dtype == "f16" and high != 1.0:
        pytest.skip("the values are not numbers of the type")
    p = Paged(70, store, 1, dim, 16, new, [400, 70, 420])
    value_scale(p, 0, 0, 200, low, False)
    value_scale(p, 0, 200, 400, high, True)
    value_scale(p, 1, 0, 70, low, False)                         # nothing else
    value_scale(p, 2, 0, 210, high, True)
    value_scale(p, 2, 210, 420, low, False)
    # held values are at most 448; scales below 2^-100 count to a step of 2^-118
    attend(p, TYPES[dtype], group, floor=448 * 2.0 ** -118)


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_zero_rows_whose_keys_win_by_little(store):
    # the zero rows' scores are 6 * log 2 below those of large values: a sixty-fourth of the sum
    p = Paged(71, store, 1, 64, 16, [2], [300], fill=False)
    k, v = torch.zeros(300, 1, 64, device=DEV), torch.randn(300, 1, 64, device=DEV)
    k[150:, 0, 0] = 1.0
    v[:150] = 0
    v[150:] *= 2.0 ** 40
    p.cache.write(k, v, prefix(p.length), p.lengths, p.d_table)
    n = 600                                                      # as many requests over the one cache: a block has whole ones
    q = torch.zeros(2 * n, 1, 64, dtype=torch.bfloat16, device=DEV)
    q[:, 0, 0] = 4.15625
    out, lse = p.cache.attend(q, prefix([2] * n), i32([300] * n), p.d_table.expand(n, -1).contiguous(), scale=1.0, lse=True)
    for i in range(0, 2 * n, 26):
        check(p, q[i:i + 2], out[i:i + 2], lse[i:i + 2], 1.0)


# ---- offsets that reach past the call's rows ----------------------------------------------------------------------------

@pytest.mark.parametrize("store,dtype", [("bf16", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("new,n,window", [([3, 6], 7, 0), ([100, 200], 250, 64), ([5, 4, 3], 5, 0)])
def test_a_token_keeps_its_position_where_the_rows_end_before_the_offsets(store, dtype, new, n, window):
    p = Paged(81, store, 2, 64, 16, new, [m + 50 for m in new])
    q = torch.randn(n, 4, 64, device=DEV).to(TYPES[dtype])
    out, lse = p.cache.attend(q, *p.tokens(), window=window, lse=True)
    check(p, q, out, lse, 0.125, window)


@pytest.mark.parametrize("window", [0, 5, 2 ** 31 - 1])
def test_offsets_that_make_no_sense_give_no_keys(window):
    # the requests' ends lie so far behind the rows that every token stands before its cache
    p = Paged(84, "bf16", 2, 64, 16, [3, 100], [60, 200])
    q = torch.randn(103, 4, 64, device=DEV).bfloat16()
    out, lse = p.cache.attend(q, i32([0, 3, 2 ** 31 - 1]), p.lengths, p.d_table, window=window, lse=True)
    assert (out[3:] == 0).all() and (lse[3:] == -math.inf).all()
    p.new = [3]
    check(p, q[:3], out[:3], lse[:3], 0.125, window if window < 2 ** 31 - 1 else 0)


# ---- no wait in vain ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,length,heads,group,dim", [([30], [20011], 2, 4, 128), ([20] * 40, [2000] * 40, 4, 4, 64), ([40] * 6, [3001] * 6, 4, 7, 128),
                                                        ([17, 70, 20, 128] * 8, [1500] * 32, 2, 4, 128)])
def test_blocks_with_a_tile_and_without_a_second_one(dtype, new, length, heads, group, dim):
    # items of at most 128 rows, several units and items a block: the second tile's warps only go along.  A wait that has missed its phase
    # takes 16 ms or more, a call like these 0.1 ms
    p = Paged(87, dtype, heads, dim, 64, new, length)
    q = torch.randn(sum(new), heads * group, dim, device=DEV).to(TYPES[dtype])
    out, lse = p.cache.attend(q, *p.tokens(), lse=True)
    check(p, q, out, lse, dim ** -0.5)
    times = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    times[0].record()
    got = [p.cache.attend(q, *p.tokens()) for _ in range(50)]
    times[1].record()
    torch.cuda.synchronize()
    assert all(torch.equal(g, out) for g in got) and times[0].elapsed_time(times[1]) < 50 * 5
