"""The paged cache and the attention over it where the first tests do not go: value scales of very different size, scores that grow
along the keys, calls of several items a block, layouts of the caller's own, offsets past the call's rows, all rows against the
definition in 64 bits on the GPU; the way from the pruning into the cache; and what is left where a wait inside the kernels gives up."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2605_02218_b200 import api, workloads
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


@pytest.mark.parametrize("store,dtype,high", [("e4m3", "f16", 1.0)] + [(s, "bf16", h) for s in ("e4m3", "int8") for h in (1.0, 2.0 ** 20, 2.0 ** 100)])
@pytest.mark.parametrize("low", [0.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -100, 2.0 ** -60])
@pytest.mark.parametrize("dim,group,new", [(64, 1, [1, 1, 1]), (128, 4, [3, 1, 70])])
def test_rows_of_zeros_and_of_large_values_in_one_cache(store, dtype, low, high, dim, group, new):
    # whole units of keys with the least scales there are, before, after and without ordinary ones: they count in the sums
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


# ---- scores that grow along the keys ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "int8")])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,group,window", [([3, 8], 4, 0), ([150, 300], 3, 0), ([300, 150], 2, 400)])
def test_references_that_move_from_unit_to_unit(dtype, store, dim, new, group, window):
    # score of key t: about c * t / 100, with a slope c of each row's own, positive and negative: accumulated rows and sums are
    # brought to new references by factors between 0 and 1, row by row at different keys
    p = Paged(72, store, 2, dim, 16, new, [900, 700])
    k = 0.3 * p.k
    t = torch.cat([torch.arange(n, device=DEV) for n in p.length]).float()
    k[:, :, 0] = t[:, None] / 100
    p.cache.write(k, p.v, prefix(p.length), p.lengths, p.d_table)
    n = sum(new)
    g = torch.Generator(device=DEV).manual_seed(6)
    q = torch.randn(n, 2 * group, dim, generator=g, device=DEV)
    q[:, :, 0] = torch.linspace(-6, 14, n * 2 * group, device=DEV).view(n, -1)[torch.randperm(n, generator=g, device=DEV)]
    q = q.to(TYPES[dtype])
    out, lse = p.cache.attend(q, *p.tokens(), scale=1.0, window=window, lse=True)
    check(p, q, out, lse, 1.0, window)


# ---- several items a block ----------------------------------------------------------------------------------------------

def steps_a_share(p, group, window, rows=256, keys=128, opening=4):
    """Places of the line of items and units that one block of the kernel for many rows takes, and the longest item's."""
    total = longest = 0
    for m, length in zip(p.new, p.length):
        for tile in range(-(-m * group // rows)):
            first, last = tile * rows, min((tile + 1) * rows, m * group) - 1
            hi = length - m + last // group + 1
            lo = max(length - m + first // group - window + 1, 0) if window else 0
            steps = opening + (hi - 1) // keys - lo // keys + 1
            total += p.heads * steps
            longest = max(longest, steps)
    return total / torch.cuda.get_device_properties(0).multi_processor_count, longest


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim,heads,group,page,window,counts", [
    (128, 4, 4, 16, 0, [512] * 12), (64, 16, 1, 64, 0, [600] * 8), (128, 8, 2, 128, 300, [512, 700, 90, 640] * 3), (64, 2, 7, 32, 512, [700, 333, 64, 901] * 4)])
def test_many_items_a_block(dtype, dim, heads, group, page, window, counts):
    # a block goes from item to item: new queries, S and O used again, the rings of units and slots several times round
    rng = np.random.default_rng(73)
    new = counts
    length = [m + int(rng.integers(0, 1100)) for m in new]
    p = Paged(74, dtype, heads, dim, page, new, length)
    share, longest = steps_a_share(p, group, window)
    assert share > 1.5 * longest and share > 12
    q, out, lse = attend(p, TYPES[dtype], heads * group, window=window)
    for _ in range(3):
        again, l = p.cache.attend(q, *p.tokens(), window=window, lse=True)
        assert torch.equal(again, out) and torch.equal(l, lse)


@pytest.mark.parametrize("store,dtype", [("e4m3", "bf16"), ("int8", "f16"), ("bf16", "bf16")])
def test_blocks_and_single_tokens_of_many_requests(store, dtype):
    rng = np.random.default_rng(75)
    length = [int(v) for v in rng.integers(300, 4000, 48)]
    p = Paged(76, store, 4, 128, 64, [int(v) for v in rng.integers(0, 9, 48)], length)
    attend(p, TYPES[dtype], 16, max_new=8)


# ---- layouts ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("store,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("page", [8, 16, 128])
def test_pages_further_apart_than_their_size(store, dtype, page):
    p = Paged(77, store, 2, 128, page, [1, 9, 130], [500, 9, 400])
    own = p.cache
    if page == 16:                                               # 16 bytes of something else between pages
        gap, size = 16 // own.k.element_size(), own.k[0].numel()
        far = [torch.zeros(p.pages * (size + gap), dtype=torch.uint8 if own.k.element_size() == 1 else torch.int16, device=DEV).view(own.k.dtype)
               .as_strided(own.k.shape, (size + gap,) + own.k.stride()[1:]) for _ in range(2)]
    else:                                                        # keys and values page by page in one allocation
        both = torch.stack([own.k.view(torch.uint8), own.v.view(torch.uint8)], 1)
        far = [both[:, i].view(own.k.dtype) for i in range(2)]
    far[0].view(torch.uint8).copy_(own.k.view(torch.uint8))
    far[1].view(torch.uint8).copy_(own.v.view(torch.uint8))
    q, out, lse = attend(p, TYPES[dtype], 6)
    p.cache = api.PagedCache(*far, *(s for s in (own.k_scale, own.v_scale) if s is not None))
    got, l = p.cache.attend(q, *p.tokens(), lse=True)
    assert torch.equal(got, out) and torch.equal(l, lse)
    for a, b in zip(p.cache.read(*p.tokens(), sum(p.new)), own.read(*p.tokens(), sum(p.new))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("store,dtype", [("bf16", "bf16"), ("int8", "f16")])
def test_a_table_with_rows_of_its_own_stride(store, dtype):
    p = Paged(78, store, 2, 64, 16, [1, 9, 130], [500, 9, 400])
    q, out, lse = attend(p, TYPES[dtype], 6)
    wide = torch.full((len(p.new), p.d_table.shape[1] + 5), 10 ** 6, dtype=torch.int32, device=DEV)
    table = wide[:, :p.d_table.shape[1]]
    table.copy_(p.d_table)
    t = p.tokens()[:2] + (table,)
    got, l = p.cache.attend(q, *t, lse=True)
    assert torch.equal(got, out) and torch.equal(l, lse)
    for a, b in zip(p.cache.read(*t, sum(p.new)), p.cache.read(*p.tokens(), sum(p.new))):
        assert torch.equal(a, b)
    before = [x.clone() for x in p.cache.read(*p.tokens(), sum(p.new))]
    kv = torch.randn(sum(p.new), 2, 2, 64, device=DEV).bfloat16()
    p.cache.write(kv[:, 0], kv[:, 1], *t)
    after = p.cache.read(*p.tokens(), sum(p.new))
    p.cache.write(kv[:, 0], kv[:, 1], *p.tokens())
    again = p.cache.read(*p.tokens(), sum(p.new))
    assert all(torch.equal(a, b) and not torch.equal(a, c) for a, b, c in zip(after, again, before))


@pytest.mark.parametrize("store,dtype", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "f16")])
@pytest.mark.parametrize("page", [512, 4096])
def test_large_pages(store, dtype, page):
    p = Paged(79, store, 2, 64, page, [1, 9, 200], [5000, 9, 700], stray_pages=1)
    attend(p, TYPES[dtype], 4)
    k, v = p.cache.read(prefix(p.length), p.lengths, p.d_table, sum(p.length), dtype=torch.float32)
    want = [torch.from_numpy(np.concatenate([p.rows(b)[i] for b in range(3)])).to(DEV) for i in range(2)]
    assert torch.equal(k, want[0].float()) and torch.equal(v, want[1].float())


@pytest.mark.parametrize("most", [1, 3, 20])
def test_more_new_tokens_than_the_hint_says(most):
    p = Paged(80, "bf16", 2, 128, 16, [300, 1, 40, 17], [900, 200, 40, 300])
    attend(p, torch.bfloat16, 8, max_new=most)
    attend(p, torch.bfloat16, 8, max_new=most, window=100)


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


@pytest.mark.parametrize("store,dtype", [("bf16", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("end", [-2 ** 31, -2 ** 31 + 3, -2 ** 31 + 100, -1, 0, 99])
def test_an_end_before_the_start_is_a_request_without_rows(store, dtype, end):
    # in 32 bits the least number less the start is a large one
    p = Paged(89, store, 2, 64, 16, [100, 0, 0], [150, 200, 30])
    q = torch.randn(120, 4, 64, device=DEV).to(TYPES[dtype])
    out = torch.full_like(q, 3.0)
    p.cache.attend(q, i32([0, 100, end, end]), p.lengths, p.d_table, out=out)
    assert (out[100:] == 3).all()
    check(p, q[:100], out[:100], None, 0.125)


# ---- from the pruning into the cache ------------------------------------------------------------------------------------

def test_the_kept_tokens_of_a_selection_go_into_the_cache():
    wl = workloads.make_workload("kept", seed=82, dtype=torch.bfloat16, batch=3, n_vis=(150, 700), n_txt=(3, 20), d=256, n_heads=2, rank=16,
                                 keep_ratio=0.25).to(DEV)
    pruner = api.Pruner.for_workload(wl)
    m = pruner.marshal(wl)
    keep_idx, ko, *_ = pruner.select(m, pruner.score(m)[2])
    kept = [int(v) for v in np.diff(ko)]
    kv = torch.randn(2, wl.total_vis, 4, 128, device=DEV).bfloat16()
    dense = [pruner.compact_rows(m, keep_idx, ko, x) for x in kv]
    pruner.close()
    got = []
    for direct in (True, False):
        p = Paged(83, "e4m3", 4, 128, 16, kept, kept, fill=False)
        if direct:
            p.cache.write(kv[0], kv[1], *p.tokens(), rows=keep_idx, row_offsets=i32(wl.vis_offsets.tolist()))
        else:
            p.cache.write(*dense, *p.tokens())
        got.append(p.cache.read(*p.tokens(), sum(kept)))
        q = torch.randn(sum(kept), 8, 128, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).bfloat16()
        out, lse = p.cache.attend(q, *p.tokens(), lse=True)
        check(p, q, out, lse, 128 ** -0.5)
    assert all(torch.equal(a, b) and a.isfinite().all() for a, b in zip(*got))


def test_an_argument_without_a_truth_value_is_refused():
    p = Paged(88, "bf16", 2, 64, 16, [3], [20])
    q = torch.randn(3, 4, 64, device=DEV).bfloat16()
    with pytest.raises(ValueError):                              # what bool() says of it
        p.cache.attend(q, *p.tokens(), lse=np.array([1, 2]))
    out, lse = p.cache.attend(q, *p.tokens(), lse=np.True_)
    check(p, q, out, lse, 0.125)
