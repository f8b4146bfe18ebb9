"""The verification operators on the GPU against their definitions in 64 bits: edits of logits, the paged cache, attention."""
import math

import numpy as np
import pytest
import torch

from oracle import verify_oracle as O
from paper_2605_02218_b200 import api

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def half(dtype):
    """A rounding to the type, relative to the value."""
    return torch.finfo(dtype).eps / 2


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prefix(counts):
    return i32(np.concatenate([[0], np.cumsum(counts)]).astype(np.int64).tolist())


# ---- edits of logits ----------------------------------------------------------------------------------------------------

def edit_case(seed, dtype, rows, vocab, hist, bias=0, mask=False, ids_past_the_end=False):
    rng = np.random.default_rng(seed)
    ld = -(-vocab // 8) * 8
    n, batch = sum(rows), len(rows)
    z = torch.from_numpy(3 * rng.standard_normal((n, ld))).to(dtype).to(DEV)
    few = max(2, vocab // 7)                                     # tokens repeat
    history = [rng.integers(0, few, h) for h in hist]
    if ids_past_the_end:
        for h in history:
            h[::3] = [-1, vocab, 2 ** 31 - 1, -2 ** 31][: 1 + int(rng.integers(4))][-1]
    c = dict(z=z, rows=rows, vocab=vocab, history=history, prompt=[int(rng.integers(0, h + 1)) for h in hist],
             drafted=rng.integers(0, few, n), repetition=1 + 0.5 * rng.random(batch), presence=rng.random(batch),
             frequency=0.3 * rng.random(batch), bias=None, allowed=None)
    for name in ("repetition", "presence", "frequency"):
        c[name] = c[name].astype(np.float32)
    if bias:
        c["bias"] = [[(int(rng.integers(0, vocab)), float(np.float32(rng.standard_normal()))) for _ in range(bias + b)] for b in range(batch)]
    if mask:
        c["allowed"] = rng.random((n, vocab)) < 0.5
    return c


def edit_args(c):
    vocab, n = c["vocab"], c["z"].shape[0]
    a = dict(history=i32(np.concatenate(c["history"]).tolist()), history_offsets=prefix([len(h) for h in c["history"]]),
             prompt_lengths=i32(c["prompt"]), drafted=i32(c["drafted"].tolist()), vocab=vocab)
    for name in ("repetition", "presence", "frequency"):
        a[name] = torch.from_numpy(c[name]).to(DEV)
    if c["bias"] is not None:
        flat = [p for b in c["bias"] for p in b]
        a.update(bias_ids=i32([p[0] for p in flat]), bias_values=torch.tensor([p[1] for p in flat], device=DEV),
                 bias_offsets=prefix([len(b) for b in c["bias"]]))
    if c["allowed"] is not None:
        bits = np.zeros((n, -(-vocab // 32) * 32), dtype=bool)
        bits[:, :vocab] = c["allowed"]
        words = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
        a["mask"] = torch.from_numpy(words.copy()).to(DEV)
    return a


def edit_check(c, out):
    dtype, vocab = c["z"].dtype, c["vocab"]
    z = c["z"][:, :vocab].double().cpu().numpy()
    got = out[:, :vocab].double().cpu().numpy()
    row = 0
    for b, n in enumerate(c["rows"]):
        first = row
        for _ in range(n):
            bias = c["bias"][b] if c["bias"] is not None else ()
            allowed = None if c["allowed"] is None else c["allowed"][row]
            want = O.edit_row(z[row], c["history"][b], c["prompt"][b], c["drafted"][first:row], float(c["repetition"][b]),
                              float(c["presence"][b]), float(c["frequency"][b]), bias, allowed)
            fine = np.isfinite(want)
            assert np.array_equal(fine, np.isfinite(got[row])) and (got[row][~fine] == -np.inf).all()
            # at most six float32 roundings of numbers no larger than the sum of all magnitudes, then one to the type
            times = len(c["history"][b]) + row - first
            size = np.abs(z[row]) * c["repetition"][b] + c["frequency"][b] * times + c["presence"][b] + max([abs(v) for _, v in bias], default=0)
            limit = 6 * 2.0 ** -24 * size + half(dtype) * np.abs(want) + 2.0 ** -25 * (dtype == torch.float16)
            assert (np.abs(got[row] - want)[fine] <= limit[fine]).all()
            row += 1


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,hist,bias,mask", [
    ([1], 2, [1], 0, False), ([1], 33, [0], 1, True), ([3, 0, 5], 1000, [10, 400, 1], 3, True), ([8], 4097, [700], 0, True),
    ([0, 2, 0, 1, 4], 12289, [30, 0, 9, 5000, 17], 40, False), ([17] * 4, 8191, [100, 1, 50, 2000], 5, True),
])
def test_edits_follow_the_definition(dtype, rows, vocab, hist, bias, mask):
    c = edit_case(hash((vocab, len(rows))) % 1000, TYPES[dtype], rows, vocab, hist, bias, mask, ids_past_the_end=vocab == 1000)
    edit_check(c, api.edit_logits(c["z"], prefix(rows), **edit_args(c)))


def test_many_rows_of_few_entries_and_few_rows_of_many():
    for rows, vocab, hist in (([3] * 200, 700, [20] * 200), ([1], 151674, [3000])):
        c = edit_case(5, torch.float16, rows, vocab, hist, 2, True)
        edit_check(c, api.edit_logits(c["z"], prefix(rows), **edit_args(c)))


def test_edits_in_place_leave_padding_and_foreign_rows():
    c = edit_case(6, torch.bfloat16, [2, 3], 1001, [50, 60], 4, True)
    want = api.edit_logits(c["z"], prefix(c["rows"]), **edit_args(c))
    z = torch.full((9, 1008), 7.0, dtype=torch.bfloat16, device=DEV)
    z[2:7] = c["z"]
    z[:, 1001:] = 7.0
    off = i32([2, 4, 7])                                          # rows 0, 1, 7, 8 belong to nobody
    a = edit_args(c)
    a["drafted"] = torch.cat([i32([0, 0]), a["drafted"], i32([0, 0])])
    a["mask"] = torch.cat([a["mask"][:2], a["mask"], a["mask"][:2]])
    got = api.edit_logits(z, off, out=z, **a)
    assert got is z and torch.equal(z[2:7, :1001], want[:, :1001])
    assert (z[:, 1001:] == 7).all() and (z[:2] == 7).all() and (z[7:] == 7).all()


def test_without_edits_every_bit_stays():
    bits = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).to(DEV).view(1, -1)
    for dtype in (torch.float16, torch.bfloat16):
        z = bits.view(dtype)                                     # every number, infinity and NaN of the type
        assert torch.equal(api.edit_logits(z, prefix([1])).view(torch.int16), bits)
        one = api.edit_logits(z, prefix([1]), history=i32([5]), history_offsets=prefix([1]), repetition=torch.full((1,), 1.2, device=DEV))
        same = torch.ones(65536, dtype=torch.bool)
        same[5] = False
        assert torch.equal(one.view(torch.int16)[0].cpu()[same], bits[0].cpu()[same])


def test_logits_that_are_not_finite():
    z = torch.tensor([[-math.inf, math.inf, math.nan, torch.finfo(torch.float32).min, 1.0, -0.0, 0.0, 2.0]], device=DEV)
    got = api.edit_logits(z, prefix([1]), history=i32(list(range(8))), history_offsets=prefix([8]), prompt_lengths=i32([8]),
                          repetition=torch.full((1,), 2.0, device=DEV), mask=i32([[0b01111111]]))[0].tolist()
    assert got[0] == -math.inf and got[1] == math.inf and math.isnan(got[2]) and got[3] == -math.inf and got[4] == 0.5
    assert got[5] == 0 and got[6] == 0 and got[7] == -math.inf


def test_a_row_whose_mask_leaves_nothing():
    z = torch.randn(2, 512, device=DEV).half()
    mask = torch.zeros(2, 16, dtype=torch.int32, device=DEV)
    mask[1, 3] = 1 << 31 >> 31 & 1
    got = api.edit_logits(z, prefix([2]), mask=mask)
    assert (got[0] == -math.inf).all() and got[1].isfinite().nonzero().flatten().tolist() == [96]
    assert torch.equal(got[1, 96], z[1, 96])


# ---- the paged cache ----------------------------------------------------------------------------------------------------

class Paged:
    """A cache, the batch's places in it, and what the oracle reads of it."""

    def __init__(self, seed, store, heads, dim, page, new, length, stray_pages=3, fill=True, holes=(), apart=False):
        rng = np.random.default_rng(seed)
        self.rng, self.store, self.heads, self.dim, self.page, self.new, self.length = rng, store, heads, dim, page, new, length
        used = [-(-v // page) for v in length]
        self.pages, width = sum(used) + stray_pages, max(used + [1]) + 1
        order = rng.permutation(self.pages)
        table = rng.choice([-1, self.pages, 2 ** 31 - 1, 0], (len(new), width))   # past the length: anything
        at = 0
        for b, u in enumerate(used):
            table[b, :u] = order[at:at + u]
            at += u
        for b, slot, page_id in holes:
            table[b, slot] = page_id
        self.table = table
        dtype = TYPES[store]
        shape = (self.pages, heads, page, dim)
        # stale memory: NaN and infinity wherever no call has written
        k = torch.full(shape, math.nan if dtype.is_floating_point else 99.0).to(dtype)
        v = torch.full(shape, math.nan if store in ("e4m3", "bf16") else math.inf if dtype.is_floating_point else 99.0).to(dtype)
        if apart:                                                # one allocation for both, page by page
            both = torch.stack([k.view(torch.uint8), v.view(torch.uint8)], 1).to(DEV)
            k, v = both[:, 0].view(dtype), both[:, 1].view(dtype)
        scales = [torch.full(shape[:3], math.nan, device=DEV) for _ in range(2)] if store in O.LARGEST else []
        self.cache = api.PagedCache(k.to(DEV), v.to(DEV), *scales)
        self.lengths, self.d_table = i32(length), i32(table.tolist())
        if fill:                                                 # all positions, by the call itself: it has its own tests
            n = sum(length)
            self.k, self.v = (torch.from_numpy(rng.standard_normal((max(n, 1), heads, dim)) * np.exp(0.3 * rng.standard_normal((max(n, 1), heads, 1)))).float().to(DEV)
                              for _ in range(2))
            self.cache.write(self.k[:n], self.v[:n], prefix(length), self.lengths, self.d_table)

    def tokens(self):
        return prefix(self.new), self.lengths, self.d_table

    def rows(self, b):
        """(k, v) [length, heads, dim] in 64 bits as held, and which positions have a place."""
        c, out = self.cache, []
        spots = [O.place(t, self.table[b], self.page, self.pages) for t in range(self.length[b])]
        there = np.array([s is not None for s in spots], dtype=bool)
        page = torch.tensor([s[0] if s else 0 for s in spots], dtype=torch.long, device=DEV)
        at = torch.tensor([s[1] if s else 0 for s in spots], dtype=torch.long, device=DEV)
        for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
            y = x[page, :, at].double()
            if s is not None:
                y = y * s[page, :, at].double()[..., None]
            out.append(np.where(there[:, None, None], y.cpu().numpy(), 0.0))
        return out[0], out[1], there


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("store", ["f32", "bf16", "f16", "e4m3", "int8"])
@pytest.mark.parametrize("heads,dim,page", [(1, 64, 8), (3, 128, 16), (8, 64, 64)])
def test_written_rows_are_held_as_defined(dtype, store, heads, dim, page):
    new, length = [3, 0, 1, 40, 2], [3, 0, 17, 45, 1]             # the last one has a token without a position
    p = Paged(1, store, heads, dim, page, new, length, fill=False, apart=True)
    n = sum(new)
    qkv = torch.randn(n + 1, 3, heads, dim, device=DEV).to(TYPES[dtype])
    qkv[0, 1] = 0                                                # a row of zeros
    qkv[1, 2] *= 1e-3
    before = [p.cache.k.view(torch.uint8).clone(), p.cache.v.view(torch.uint8).clone()]
    p.cache.write(qkv[:n, 1], qkv[:n, 2], *p.tokens())
    touched = torch.zeros(p.pages, heads, page, dtype=torch.bool)
    i = 0
    for b, m in enumerate(new):
        for j in range(m):
            spot = O.place(length[b] - m + j, p.table[b], page, p.pages)
            for x, s, src in ((p.cache.k, p.cache.k_scale, qkv[i, 1]), (p.cache.v, p.cache.v_scale, qkv[i, 2])):
                if spot is None:
                    continue
                touched[spot[0], :, spot[1]] = True
                got = x[spot[0], :, spot[1]]
                if s is None:
                    assert torch.equal(got, src.to(TYPES[store]))
                else:
                    want, scale = O.held(src.double().cpu().numpy(), store)
                    assert np.array_equal(s[spot[0], :, spot[1]].cpu().numpy(), scale)
                    assert np.array_equal(got.double().cpu().numpy(), want)
            i += 1
    assert int(touched.sum()) == (n - 1) * heads
    for x, old in ((p.cache.k, before[0]), (p.cache.v, before[1])):   # nothing else was touched
        same = (x.view(torch.uint8) == old).all(-1).cpu()
        assert same[~touched].all()


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_quotients_next_to_a_border_round_the_right_way(store, dtype):
    # rows whose values lie at, just above and just below the borders between two held values
    rng = np.random.default_rng(3)
    n, dim, most = 600, 128, O.LARGEST[store]
    top = torch.from_numpy(np.exp(rng.uniform(-9, 9, n))).to(TYPES[dtype]).double().numpy()
    scale = (top / most).astype(np.float32).astype(np.float64)
    if store == "int8":
        border = rng.integers(0, 127, (n, dim)) + 0.5
    else:
        m = np.ldexp(rng.integers(8, 16, (n, dim)) + 0.5, rng.integers(-9, 6, (n, dim)))
        border = np.minimum(m, 440.0)
    x = torch.from_numpy(border * scale[:, None] * rng.choice([-1, 1], (n, dim)))
    x = x.to(TYPES[dtype])
    off = rng.integers(-1, 2, (n, dim))
    bits = x.view(torch.int32 if dtype == "f32" else torch.int16)
    x = (bits + torch.from_numpy(off).to(bits.dtype)).view(TYPES[dtype])   # a step of the type up or down
    x = torch.where(x.double().abs() > torch.from_numpy(top)[:, None], torch.zeros_like(x), x)
    x[:, 0] = torch.from_numpy(top).to(TYPES[dtype])
    x = x.view(n, 1, dim).to(DEV)
    cache = api.PagedCache.empty(n // 8 + 1, 1, 8, dim, TYPES[store])
    cache.write(x, x.flip(0).contiguous(), i32([0, n]), i32([n]), torch.arange(n // 8 + 1, dtype=torch.int32, device=DEV)[None])
    want, s = O.held(x.double().cpu().numpy()[:, 0], store)
    got = cache.k.view(-1, dim)[:n].double().cpu().numpy()
    # a step down from a float16 zero is a NaN: such a row is marked by its scale
    assert np.array_equal(cache.k_scale.view(-1)[:n].cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(got[~np.isnan(s)], want[~np.isnan(s)]) and np.isnan(s).mean() < 0.5


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_rows_at_the_ends_of_the_range(store):
    rows = torch.zeros(7, 1, 64, device=DEV)
    rows[0] = 3e38
    rows[1, 0, :5] = torch.tensor([1e-38, -1e-40, 1e-45, 0, 3e-39])   # below the least scale's reach
    rows[2, 0, 3] = math.inf
    rows[3, 0, 60] = math.nan
    rows[4, 0, 7] = -math.inf
    rows[5, 0, :2] = torch.tensor([1e-28, -5e-29])
    rows[6, 0, 1] = 1.0
    cache = api.PagedCache.empty(1, 1, 8, 64, TYPES[store])
    t = i32([0, 7]), i32([7]), i32([[0]])
    cache.write(rows, rows, *t)
    for i in (0, 1, 5, 6):
        want, s = O.held(rows[i].double().cpu().numpy(), store)
        assert float(cache.k_scale[0, 0, i]) == float(s[0]) and np.array_equal(cache.k[0, :, i].double().cpu().numpy(), want)
    k, v = cache.read(*t, 7, dtype=torch.float32)
    for i in (2, 3, 4):
        assert k[i].isnan().all() and v[i].isnan().all()
    assert k[[0, 1, 5, 6]].isfinite().all()


@pytest.mark.parametrize("store", ["f32", "bf16", "f16", "e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,dim,page", [(2, 128, 16), (5, 64, 8)])
def test_read_gives_what_is_held(store, dtype, heads, dim, page):
    p = Paged(4, store, heads, dim, page, [5, 0, 30, 1], [9, 3, 30, 80], holes=[(2, 1, -1), (2, 0, 10 ** 6)])
    n = sum(p.new)
    k, v = p.cache.read(*p.tokens(), n, dtype=TYPES[dtype])
    i = 0
    for b, m in enumerate(p.new):
        kk, vv, _ = p.rows(b)
        for x, y in ((k, kk), (v, vv)):
            want = y[p.length[b] - m:]
            got = x[i:i + m].double().cpu().numpy()
            # value * scale in float32, then to the type (float16 also has its subnormal step)
            limit = np.abs(want) * (2.0 ** -24 * (store in O.LARGEST) + half(TYPES[dtype]) * (dtype != "f32") * 1.01) + 2.0 ** -25 * (dtype == "f16")
            assert (np.abs(got - want) <= limit).all()
        i += m


def test_kept_rows_go_from_a_prefill_into_the_cache():
    # the rows that a selection keeps, ascending inside each request: what compact_rows would gather
    rng = np.random.default_rng(8)
    vis, keep = [50, 7, 300], [9, 7, 41]
    idx = [np.sort(rng.choice(n, k, replace=False)) for n, k in zip(vis, keep)]
    kv = torch.randn(sum(vis), 2, 4, 128, device=DEV).bfloat16()
    off = prefix(vis)
    rows = i32(np.concatenate(idx).tolist())
    flat = torch.cat([torch.from_numpy(i) + o for i, o in zip(idx, np.concatenate([[0], np.cumsum(vis)]))]).to(DEV)
    made = []
    for direct in (True, False):
        p = Paged(9, "int8", 4, 128, 16, keep, keep, fill=False)
        if direct:
            p.cache.write(kv[:, 0], kv[:, 1], *p.tokens(), rows=rows, row_offsets=off)
        else:
            p.cache.write(kv[flat, 0], kv[flat, 1], *p.tokens())
        made.append([x.clone() for x in p.cache.read(*p.tokens(), sum(keep))])
    assert torch.equal(made[0][0], made[1][0]) and torch.equal(made[0][1], made[1][1])
    # rows that the prefill does not have are passed over
    p = Paged(9, "int8", 4, 128, 16, keep, keep, fill=False)
    bad = rows.clone()
    bad[3], bad[20] = -60, 10 ** 9
    p.cache.write(kv[:, 0], kv[:, 1], *p.tokens(), rows=bad, row_offsets=off)
    k, _ = p.cache.read(*p.tokens(), sum(keep))
    assert k[[3, 20]].isnan().all() and k[[2, 4, 19, 21]].isfinite().all()


# ---- attention ----------------------------------------------------------------------------------------------------------

def attend_check(p, q, out, lse, scale, window, skip=()):
    dtype, n_i = q.dtype, 0
    group = q.shape[1] // p.heads
    qd, od = q.double().cpu().numpy(), out.double().cpu().numpy()
    ld = None if lse is None else lse.double().cpu().numpy()
    for b, m in enumerate(p.new):
        if m == 0:
            continue
        k, v, there = p.rows(b)
        for j in range(m):
            pos = p.length[b] - m + j
            for h in range(q.shape[1]):
                want, log, size, reach = O.attend_row(qd[n_i, h], pos, k[:, h // group], v[:, h // group], there, scale, window)
                # scores: dim products summed in float32 (2^-23 a step, whatever the order) and two more roundings;
                # probabilities: one rounding to the type, the exponential and the sums in float32
                ds = (p.dim + 4) * 2.0 ** -23 * reach
                keys = max(len(k), 1)
                limit = size * (half(dtype) * 1.01 + 2 * ds + (keys + 64) * 2.0 ** -23) + half(dtype) * np.abs(want) * 1.01
                # float16 below 2^-14: a fixed step, in every probability (the largest product with a value's scale is 1) and the row
                limit += 2.0 ** -25 * (dtype == torch.float16) * (1 + keys * np.abs(v).max(initial=0))
                off = np.abs(od[n_i, h] - want)
                assert (off <= limit).all(), (b, j, h, float((off / limit.clip(1e-30)).max()))
                if ld is not None:
                    if log == -np.inf:
                        assert ld[n_i, h] == -np.inf
                    else:
                        assert abs(ld[n_i, h] - log) <= ds + (keys + 64) * 2.0 ** -23 + 2.0 ** -22 * abs(log), (b, j, h)
            n_i += 1


def attend(p, dtype, q_heads, window=0, scale=None, seed=11, **kw):
    n = sum(p.new)
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randn(n, q_heads, p.dim, generator=g, device=DEV).to(dtype)
    out, lse = p.cache.attend(q, *p.tokens(), scale=scale, window=window, lse=True, **kw)
    attend_check(p, q, out, lse, scale if scale is not None else p.dim ** -0.5, window)
    return q, out, lse


KINDS = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3"), ("bf16", "int8"), ("f16", "int8")]


@pytest.mark.parametrize("dtype,store", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 7])
def test_single_tokens(dtype, store, dim, group):
    p = Paged(20, store, 2, dim, 16, [1, 1, 0, 1, 1, 1], [1, 2, 5, 64, 65, 300])
    attend(p, TYPES[dtype], 2 * group, max_new=1)


@pytest.mark.parametrize("dtype,store", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group,page", [(1, 8, 8), (3, 2, 32), (2, 1, 128)])
def test_blocks_of_every_size(dtype, store, dim, heads, group, page):
    new, length = [3, 1, 0, 8, 17, 5], [3, 130, 9, 100, 17, 64]
    p = Paged(21, store, heads, dim, page, new, length)
    attend(p, TYPES[dtype], heads * group, max_new=17)


@pytest.mark.parametrize("dtype,store", KINDS)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 8), (128, 256)])
def test_chunks_of_prompts(dtype, store, dim, page):
    p = Paged(22, store, 1, dim, page, [150, 2, 333], [150, 200, 400])
    attend(p, TYPES[dtype], 3)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f16", "int8"), ("bf16", "e4m3")])
@pytest.mark.parametrize("new,length", [([5], [3]), ([1], [0]), ([4, 2, 1], [0, 5, 0]), ([70], [1]), ([200, 1], [131, 0])])
def test_tokens_without_a_key(dtype, store, new, length):
    # more new tokens than positions: the first ones stand before the cache and see nothing
    p = Paged(23, store, 2, 64, 8, new, length)
    for most in (0, max(new)):
        _, out, lse = attend(p, TYPES[dtype], 4, max_new=most)
        lost = new[0] - length[0]
        assert (out[:lost] == 0).all() and (lse[:lost] == -math.inf).all()


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "int8")])
@pytest.mark.parametrize("window", [1, 7, 64, 100, 2 ** 31 - 1])
def test_windows(dtype, store, window):
    p = Paged(24, store, 2, 64, 16, [1, 9, 130, 3], [500, 9, 400, 70])
    attend(p, TYPES[dtype], 6, window=window)


@pytest.mark.parametrize("dtype,store", [("bf16", "bf16"), ("f16", "e4m3")])
def test_positions_without_a_page_are_not_attended_to(dtype, store):
    p = Paged(25, store, 2, 128, 16, [4, 20, 1], [100, 90, 40], holes=[(0, 2, -1), (1, 0, 2 ** 31 - 1), (1, 4, 10 ** 6), (2, 0, -7), (2, 1, -1), (2, 2, -1)])
    _, out, lse = attend(p, TYPES[dtype], 4)
    assert (out[-1] == 0).all() and (lse[-1] == -math.inf).all()
    # a table shorter than the length: what lies past it has no place
    short = p.d_table[:, :2].contiguous()
    q = torch.randn(25, 4, 128, device=DEV).to(TYPES[dtype])
    got = p.cache.attend(q, prefix(p.new), p.lengths, short)
    p.table = p.table[:, :2]
    attend_check(p, q, got, None, 128 ** -0.5, 0)


@pytest.mark.parametrize("heads,q_heads,new", [(1, 1, 1), (2, 14, 1), (1, 8, 6), (2, 8, 30)])
def test_one_long_cache_is_cut_among_all_processors(heads, q_heads, new):
    p = Paged(26, "bf16", heads, 128, 64, [new], [20011])
    attend(p, torch.bfloat16, q_heads, max_new=new)


def test_many_requests_of_uneven_length():
    rng = np.random.default_rng(2)
    length = [int(v) for v in np.exp(rng.uniform(0, 7, 300))]
    new = [int(rng.integers(0, min(v, 4) + 1)) for v in length]
    p = Paged(27, "int8", 2, 64, 16, new, length)
    attend(p, torch.bfloat16, 4)


def test_extreme_scores_and_scales():
    p = Paged(28, "f16", 1, 64, 16, [3, 40], [50, 60])
    attend(p, torch.float16, 2, scale=30.0)                      # the softmax picks single keys
    attend(p, torch.float16, 2, scale=0.0)
    attend(p, torch.float16, 2, scale=-1.0)
    # values of very different size in one 8-bit cache, some rows zero
    for store in ("e4m3", "int8"):
        p = Paged(29, store, 1, 64, 16, [3, 40], [50, 60], fill=False)
        v = torch.randn(110, 1, 64, device=DEV) * torch.exp(6 * torch.randn(110, 1, 1, device=DEV))
        v[::7] = 0
        p.cache.write(torch.randn(110, 1, 64, device=DEV), v, prefix(p.length), p.lengths, p.d_table)
        attend(p, torch.bfloat16, 2)


def test_a_row_that_is_not_finite_reaches_only_its_request():
    p = Paged(30, "int8", 1, 64, 16, [1, 1, 20], [40, 40, 60])
    k, v = p.k.clone(), p.v.clone()
    k[45, 0, 3] = math.nan                                       # request 1, position 5
    p.cache.write(k, v, prefix(p.length), p.lengths, p.d_table)
    q = torch.randn(22, 2, 64, device=DEV).bfloat16()
    out, lse = p.cache.attend(q, *p.tokens(), lse=True)
    assert out[1].isnan().all() and lse[1].isnan().all()
    assert out[[0] + list(range(2, 22))].isfinite().all()


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_a_value_that_is_not_finite_leaves_the_sum(store):
    # the keys are in order: the rows are NaN, their log-sums are not
    p = Paged(33, store, 1, 128, 16, [1, 2], [300, 40])
    v = p.v.clone()
    v[7, 0, 5] = math.inf
    q = torch.randn(3, 4, 128, device=DEV).half()
    _, want = p.cache.attend(q, *p.tokens(), lse=True)
    p.cache.write(p.k, v, prefix(p.length), p.lengths, p.d_table)
    out, lse = p.cache.attend(q, *p.tokens(), lse=True)
    assert out[0].isnan().all() and out[1:].isfinite().all()
    # the reference moves by one key's exponent at most: float32 sums of 300 positive numbers, 2^-23 each
    assert ((lse - want).abs() <= 364 * 2.0 ** -23 + 2.0 ** -22 * want.abs()).all()


def test_rows_strides_and_outputs_of_the_callers_own():
    p = Paged(31, "bf16", 2, 128, 16, [3, 70], [40, 200])
    n = 73
    qkv = torch.randn(n + 4, 8 + 4, 128, device=DEV).bfloat16()
    q = qkv[:n, :8]                                              # columns of one projection
    want = p.cache.attend(q.contiguous(), *p.tokens())
    big = torch.full((n + 4, 2, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    got = p.cache.attend(qkv[:, :8], *p.tokens(), out=big[:, 1])  # four tokens of no request
    assert torch.equal(got[:n], want) and (big[n:] == 7).all() and (big[:, 0] == 7).all()


def test_results_do_not_depend_on_the_hint_or_the_run():
    p = Paged(32, "e4m3", 2, 128, 16, [5, 1, 9], [700, 33, 90])
    q, out, lse = attend(p, torch.bfloat16, 8)
    for most in (1, 5, 9, 1000):
        got, l = p.cache.attend(q, *p.tokens(), max_new=most, lse=True)
        attend_check(p, q, got, l, 128 ** -0.5, 0)
    for _ in range(20):
        again, l = p.cache.attend(q, *p.tokens(), lse=True)
        assert torch.equal(again, out) and torch.equal(l, lse)


def test_places_past_32_bits():
    # 8-bit pages of 128 positions x 8 heads x 128 features: page 16500 starts behind 2^31 elements
    pages, width = 16600, 3
    k = torch.empty(pages, 8, 128, 128, dtype=torch.int8, device=DEV)
    v = torch.empty_like(k)
    cache = api.PagedCache(k, v, *(torch.ones(pages, 8, 128, device=DEV) for _ in range(2)))
    table = i32([[16599, 16450, 5], [0, 16598, 16385]])
    x = torch.randn(2 * 300, 2, 8, 128, device=DEV).bfloat16()
    t = i32([0, 300, 600]), i32([300, 300]), table
    cache.write(x[:, 0], x[:, 1], *t)
    small = api.PagedCache.empty(6, 8, 128, 128, torch.int8)
    t2 = t[0], t[1], i32([[0, 1, 2], [3, 4, 5]])
    small.write(x[:, 0], x[:, 1], *t2)
    q = torch.randn(600, 16, 128, device=DEV).bfloat16()
    for a, b in ((cache.read(*t, 600), small.read(*t2, 600)), (cache.attend(q, *t, lse=True), small.attend(q, *t2, lse=True))):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert width == table.shape[1]


# ---- used together, on streams and in graphs ----------------------------------------------------------------------------

def verify_step(s):
    """What a server does with the drafted blocks of a batch: the new keys and values into the cache, attention, a projection to
    logits, their edits, the correction."""
    p = s["p"]
    p.cache.write(s["k"], s["v"], *s["t"])
    h = p.cache.attend(s["q"], *s["t"], max_new=s["most"])
    z = h.flatten(1) @ s["head"]
    z = api.edit_logits(z, s["t"][0], **s["edits"])
    return (h, z) + tuple(api.correct(s["draft"], z, s["u"], 0.02, s["edits"]["drafted"], vocab=s["edits"]["vocab"]))


def verify_state(seed, store="int8"):
    new, length = [4, 1, 0, 6], [40, 9, 0, 130]
    p = Paged(seed, store, 2, 64, 16, new, length)
    g = torch.Generator(device=DEV).manual_seed(seed)
    n, vocab, q_heads = sum(new), 4000, 4
    c = edit_case(seed, torch.bfloat16, new, vocab, [30, 5, 0, 200], 6, True)
    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV).bfloat16()
    return dict(p=p, t=p.tokens(), most=6, q=randn(n, q_heads, 64), k=randn(n, 2, 64), v=randn(n, 2, 64),
                head=randn(q_heads * 64, vocab) / 4, draft=randn(n, vocab), edits=edit_args(c), case=c,
                u=torch.rand(n, generator=g, device=DEV))


def test_the_step_as_a_whole():
    from oracle import correction_oracle  # noqa: F401  (its own tests compare correct with it)
    s = verify_state(40)
    h, z, margin, gate, accept, mass, token = verify_step(s)
    attend_check(s["p"], s["q"], h, None, 0.125, 0)
    c = dict(s["case"], z=h.flatten(1) @ s["head"])
    edit_check(c, z)
    allowed = torch.from_numpy(c["allowed"]).to(DEV)
    assert allowed[torch.arange(len(token)), token.long()].all()  # a corrected token is one that the grammar allows
    assert ((accept >= 0) & (accept <= 1)).all() and margin.isfinite().all()


def test_two_captured_steps_and_an_eager_one():
    states = [verify_state(s, store) for s, store in ((41, "int8"), (42, "bf16"))]
    want = [[x.clone() for x in verify_step(s)] for s in states]
    graphs, outs = [], []
    for s in states:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            verify_step(s)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(verify_step(s))
        graphs.append(g)
    side = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):                                          # both at once, with eager calls beside them
        for g, st in zip(graphs, side):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                g.replay()
        p = Paged(43, "bf16", 2, 64, 16, [3], [500])
        attend(p, torch.bfloat16, 4)
    torch.cuda.synchronize()
    for got, exp in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, exp))
    # new lengths in the same memory: the replayed step follows them
    s = states[0]
    s["p"].lengths.copy_(i32([39, 9, 0, 131]))
    s["p"].length = [39, 9, 0, 131]
    graphs[0].replay()
    torch.cuda.synchronize()
    attend_check(s["p"], s["q"], outs[0][0], None, 0.125, 0)


def test_calls_on_two_streams_do_not_meet():
    states = [verify_state(s) for s in (44, 45)]
    want = [[x.clone() for x in verify_step(s)] for s in states]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        got = []
        for s, st in zip(states, side):
            with torch.cuda.stream(st):
                got.append(verify_step(s))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


# ---- refusals -----------------------------------------------------------------------------------------------------------

def test_the_binding_refuses_memory_that_the_kernels_must_not_touch():
    p = Paged(50, "int8", 2, 64, 16, [3, 4], [20, 30])
    off, lengths, table = p.tokens()
    q, kv = torch.randn(7, 4, 64, device=DEV).half(), torch.randn(7, 2, 64, device=DEV).half()
    good = dict(q=q, offsets=off, lengths=lengths, table=table)
    for error, kw in [(TypeError, dict(q=q.double())), (ValueError, dict(q=q.cpu())), (ValueError, dict(q=q[0])),
                      (ValueError, dict(q=q[:, :, ::2])), (ValueError, dict(q=q[:, :, :32].contiguous())), (TypeError, dict(offsets=off.long())),
                      (ValueError, dict(offsets=off[:2])), (ValueError, dict(lengths=lengths.cpu())), (TypeError, dict(lengths=[20, 30])),
                      (TypeError, dict(table=table.long())), (ValueError, dict(table=table[:1])), (ValueError, dict(table=table.t().contiguous().t())),
                      (ValueError, dict(out=q[:5].clone())), (TypeError, dict(out=q.bfloat16())), (ValueError, dict(window=2 ** 31))]:
        with pytest.raises(error):
            p.cache.attend(**{**good, **kw})
    for kw in (dict(window=-1), dict(max_new=-2), dict(scale=math.nan)):
        with pytest.raises(api.CovspecError):
            p.cache.attend(**good, **kw)
    with pytest.raises(api.CovspecError):
        p.cache.attend(q[:, :3].contiguous(), off, lengths, table)    # 3 query heads for 2 key heads
    for error, kw in [(TypeError, dict(k=kv.double())), (ValueError, dict(v=kv[:6])), (TypeError, dict(v=kv.float())),
                      (ValueError, dict(k=kv[:, :1])), (ValueError, dict(rows=i32([0] * 7))), (ValueError, dict(k=kv.transpose(1, 2)))]:
        with pytest.raises(error):
            p.cache.write(**{**dict(k=kv, v=kv, offsets=off, lengths=lengths, table=table), **kw})
    with pytest.raises(TypeError):
        p.cache.read(off, lengths, table, 7, dtype=torch.int8)
    with pytest.raises(ValueError):
        api.PagedCache(p.cache.k, p.cache.v)                     # no scales
    with pytest.raises(ValueError):
        api.PagedCache(p.cache.k, p.cache.v, p.cache.k_scale, p.cache.v_scale[:1])
    with pytest.raises(ValueError):
        api.PagedCache(p.cache.k.transpose(1, 2), p.cache.v.transpose(1, 2), p.cache.k_scale, p.cache.v_scale)
    with pytest.raises(api.CovspecError):
        Paged(51, "bf16", 1, 64, 16, [1], [5]).cache.attend(torch.randn(1, 1, 64, device=DEV).half(), i32([0, 1]), i32([5]), i32([[0]]))
    z = torch.zeros(3, 64, device=DEV)
    for error, kw in [(TypeError, dict(row_offsets=prefix([3]).long())), (ValueError, dict(row_offsets=prefix([3]).cpu())),
                      (ValueError, dict(out=z[:2].clone())), (TypeError, dict(out=z.half())), (ValueError, dict(history=i32([1]))),
                      (ValueError, dict(drafted=i32([1, 2]))), (TypeError, dict(repetition=torch.ones(1, device=DEV).double())),
                      (ValueError, dict(bias_ids=i32([1]))), (ValueError, dict(mask=i32([[0, 0]]))),
                      (ValueError, dict(mask=i32([[0]] * 3))), (TypeError, dict(mask=torch.zeros(3, 2, device=DEV)))]:
        with pytest.raises(error):
            api.edit_logits(z, **{**dict(row_offsets=prefix([3])), **kw})
    with pytest.raises(ValueError):
        api.edit_logits(z[:, ::2], prefix([3]))


def test_without_the_native_part_the_calls_give_the_same(monkeypatch):
    states = [verify_state(s, store) for s, store in ((60, "e4m3"), (61, "bf16"))]
    def calls():
        got = []
        for s in states:
            got += list(verify_step(s)) + list(s["p"].cache.read(*s["t"], len(s["u"]), dtype=torch.float16))
            got += list(s["p"].cache.attend(s["q"], *s["t"], window=7, lse=True))
        return got
    want = [x.clone() for x in calls()]
    monkeypatch.setattr(api, "_native", None)
    assert all(torch.equal(a, b) for a, b in zip(want, calls()))


def test_prompts_and_steps_of_many_requests_in_one_call():
    # both kernels share the call; several items a share, the ring round many times
    rng = np.random.default_rng(12)
    length = [int(v) for v in rng.integers(200, 1500, 12)]
    new = [int(min(v, rng.choice([1, 4, 40, 300]))) for v in length]
    for store, dtype in (("bf16", torch.bfloat16), ("f16", torch.float16), ("int8", torch.float16)):
        p = Paged(62, store, 2, 64, 32, new, length)
        g = torch.Generator(device=DEV).manual_seed(3)
        q = torch.randn(sum(new), 14, 64, generator=g, device=DEV).to(dtype)
        first, lse = p.cache.attend(q, *p.tokens(), window=256, lse=True)
        for _ in range(300):                                     # calls back to back
            got, l = p.cache.attend(q, *p.tokens(), window=256, lse=True)
        assert torch.equal(got, first) and torch.equal(l, lse)
        keep = [b for b, m in enumerate(new) if m <= 4]          # the oracle is slow: the short ones, row by row
        at = np.concatenate([[0], np.cumsum(new)])
        for b in keep:
            small = Paged.__new__(Paged)
            small.__dict__.update(p.__dict__, new=[0] * b + [new[b]] + [0] * (len(new) - b - 1))
            attend_check(small, q[at[b]:at[b + 1]], first[at[b]:at[b + 1]], lse[at[b]:at[b + 1]], 0.125, 256)


def test_empty_calls():
    p = Paged(52, "bf16", 2, 64, 16, [0, 0], [20, 30])
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    p.cache.write(e, e, *p.tokens())
    assert p.cache.attend(e, *p.tokens()).shape == (0, 2, 64) and p.cache.read(*p.tokens(), 0)[0].shape == (0, 2, 64)
    assert api.edit_logits(torch.empty(0, 64, device=DEV), i32([0, 0])).shape == (0, 64)
