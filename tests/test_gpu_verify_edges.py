"""The attention over the paged cache where value scales are of very different size and where offsets reach past the call's rows: all
rows against the definition in 64 bits, on the GPU.  And what it leaves where a wait inside its kernels gives up."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2605_02218_b200 import api
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


# ---- waits that give up -------------------------------------------------------------------------------------------------

def shares(p, group, window, rows, keys, opening, ctas, over=0, upto=2 ** 31 - 1):
    """For each block, (request, head, tile) of every unit of its share: the line of items and units, cut into equal shares."""
    line = []
    for b, (m, length) in enumerate(zip(p.new, p.length)):
        n = m * group
        if not over < n <= upto:
            continue
        items = []
        for tile in range(-(-n // rows)):
            first, last = tile * rows, min((tile + 1) * rows, n) - 1
            hi = max(min(length - m + last // group + 1, length), 0)
            lo = max(length - m + first // group - window + 1, 0) if window else 0
            items.append((hi - 1) // keys - lo // keys + 1 if hi > lo else 1)
        line += [x for h in range(p.heads) for t, u in enumerate(items) for x in [None] * opening + [(b, h, t)] * u]
    per = max(-(-len(line) // ctas), 1)
    return [[x for x in line[i * per:(i + 1) * per] if x is not None] for i in range(ctas)]


def kernels_of(p, dtype, q_heads, window, most):
    """Shares of the kernel for few rows and, where it runs, of the one for many; rows of their items."""
    sms, group, n = torch.cuda.get_device_properties(0).multi_processor_count, q_heads // p.heads, sum(p.new)
    top = (min(most, n) if most else n) * group
    rows = 16 if top <= 16 else 32 if top <= 32 else 64
    held = p.store in ("e4m3", "int8")
    both = top > 64 and not held

    def ctas(rows, keys, most):
        return min(most, (n * group // rows + len(p.new)) * p.heads * (-(-p.table.shape[1] * p.page // keys) + 1))
    few = shares(p, group, window, rows, 128 if held and rows < 64 else 64, 2, ctas(rows, 64, 2 * sms), 0, 64 if both else 2 ** 31 - 1)
    got = [(few, rows)]
    if both:
        got.append((shares(p, group, window, 256, 128, 4, ctas(256, 128, sms), 64), 256))
    return got


def selftest(p, q, window, most, block, unit):
    """The call with waits that give up; its scratch holds plausible numbers before."""
    n, heads = q.shape[:2]
    out = torch.full_like(q, 3.0)
    lse = torch.full((n, heads), 3.0, device=DEV)
    lib = api.load_library()
    size = lib.covspec_cache_attend_workspace(p.cache._ref, heads)
    work = torch.ones(size // 4, device=DEV)
    st = lib.covspec_selftest_attend_timeout(p.cache._ref, C.byref(p.cache._tokens(*p.tokens())), api._LOGIT_DTYPES[q.dtype], n, q.data_ptr(),
                                             heads * p.dim, heads, p.dim ** -0.5, window, most, out.data_ptr(), heads * p.dim,
                                             lse.data_ptr(), work.data_ptr(), size, block, unit, api._raw_stream())
    assert st == 0
    torch.cuda.synchronize()
    return out, lse


GIVEN_UP = [("bf16", "bf16", 128, [1, 4, 0, 2], [3000, 900, 70, 2000], 2, 0, 4),
            ("bf16", "bf16", 64, [1, 4, 0, 2] * 10, [3000, 1900, 70, 5000] * 10, 2, 0, 4),
            ("bf16", "e4m3", 128, [1, 4, 2] * 16, [3000, 900, 6000] * 16, 2, 0, 4), ("f16", "int8", 64, [40, 130] * 5, [800, 1900] * 5, 3, 0, 0),
            ("bf16", "bf16", 128, [300, 1, 700] * 4, [2500, 900, 3800] * 4, 4, 0, 0), ("f16", "f16", 64, [90, 400], [2500, 1000], 3, 500, 0)]


@pytest.mark.parametrize("dtype,store,dim,new,length,group,window,most", GIVEN_UP)
def test_rows_are_nan_where_every_wait_gives_up(dtype, store, dim, new, length, group, window, most):
    p = Paged(85, store, 2, dim, 16, new, length)
    q = torch.randn(sum(new) + 2, 2 * group, dim, device=DEV).to(TYPES[dtype])
    want = p.cache.attend(q, *p.tokens(), window=window, max_new=most, lse=True)
    out, lse = selftest(p, q, window, most, -1, 0)
    n = sum(new)
    assert out[:n].isnan().all() and lse[:n].isnan().all() and (out[n:] == 3).all() and (lse[n:] == 3).all()
    again = p.cache.attend(q, *p.tokens(), window=window, max_new=most, lse=True)
    assert all(torch.equal(a[:n], b[:n]) for a, b in zip(want, again))


@pytest.mark.parametrize("dtype,store,dim,new,length,group,window,most", GIVEN_UP)
def test_the_rows_that_a_block_had_a_part_of_are_nan_where_its_waits_give_up(dtype, store, dim, new, length, group, window, most):
    p = Paged(86, store, 2, dim, 16, new, length)
    heads, n = 2 * group, sum(new)
    q = torch.randn(n, heads, dim, device=DEV).to(TYPES[dtype])
    want = p.cache.attend(q, *p.tokens(), window=window, max_new=most, lse=True)
    kernels = kernels_of(p, dtype, heads, window, most)
    at = np.concatenate([[0], np.cumsum(new)])
    used = sorted({i for ks, _ in kernels for i, s in enumerate(ks) if s})
    cut = 0
    for block in sorted({0} | {used[len(used) * i // 5] for i in range(5)} | {used[-1]}):
        for unit in (0, 1, 3, 9):
            lost = torch.zeros(n, heads, dtype=torch.bool, device=DEV)
            for ks, rows in kernels:
                if block >= len(ks) or unit >= len(ks[block]):
                    continue
                cut += any(len({i for i, s in enumerate(ks) if item in s}) > 1 for item in set(ks[block]))
                for b, h, tile in set(ks[block]):
                    r = torch.arange(tile * rows, min((tile + 1) * rows, new[b] * group), device=DEV)
                    lost[at[b] + r // group, h * group + r % group] = True
            out, lse = selftest(p, q, window, most, block, unit)
            assert torch.equal(out.isnan().all(-1), lost) and torch.equal(lse.isnan(), lost), (block, unit)
            assert torch.equal(out[~lost], want[0][~lost]) and torch.equal(lse[~lost], want[1][~lost])
    assert cut                                                   # items that several blocks share were among them


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
