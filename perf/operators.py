"""The verification step of drafted blocks: what is measured of the operators around covspec_correct.

A server that verifies drafted blocks writes the keys and values of the new tokens (or of the visual tokens that the
pruning kept) into a paged cache, which holds them as they are or in 8 bits; attends from the new tokens over that cache;
and edits the logits of the block (penalties, biases, grammar masks) before it corrects it.  A case's "op" names the call:
  edit     api.edit_logits
  write    api.PagedCache.write
  read     api.PagedCache.read
  attend   api.PagedCache.attend

Sizes: the vocabulary, the heads and widths (12, 16, 28 and 32 heads of 128), the token counts and keep ratios of the
framework's own configurations and benchmarks; grouped key heads, page sizes and cache lengths are generic.  What belongs
to a case's sizes (lengths of a ragged batch) is drawn from its "sizes", the contents from the seed given to `prepare`.
"""
import math
import random

import torch

own = False

VOCAB = 151674
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "int8": 1}
LARGEST = {"e4m3": 448.0, "int8": 127.0}
LEAST_SCALE = 2.0 ** -100


def listed():
    return [
        # the block of one interactive session: latency
        dict(name="edit_block", op="edit", dtype="f16", batch=1, block_lo=8, block_hi=8, vocab=VOCAB, hist_lo=800, hist_hi=800,
             bias=16, mask=True, sizes=0),
        # the blocks of many sessions in one call, all of them under a grammar
        dict(name="edit_many", op="edit", dtype="f16", batch=128, block_lo=8, block_hi=8, vocab=VOCAB, hist_lo=200, hist_hi=3000,
             bias=32, mask=True, sizes=1),
        # blocks of different lengths (some sessions have none), long histories, penalties and biases alone
        dict(name="edit_ragged", op="edit", dtype="bf16", batch=48, block_lo=0, block_hi=12, vocab=92553, hist_lo=1, hist_hi=20000,
             bias=300, mask=False, sizes=2),
        # the drafted blocks of 32 sessions go into an 8-bit cache
        dict(name="write_draft", op="write", dtype="bf16", store="e4m3", batch=32, new_lo=8, new_hi=8, len_lo=300, len_hi=4096,
             heads=8, dim=128, page=16, kept=0.0, sizes=3),
        # the visual tokens that the pruning kept of ragged images (a fifth), straight from the prefill's keys and values
        dict(name="write_kept", op="write", dtype="bf16", store="int8", batch=64, new_lo=256, new_hi=4096, len_lo=0, len_hi=0,
             heads=8, dim=128, page=64, kept=0.2, sizes=4),
        # one request's cache comes back as dense rows
        dict(name="read_one", op="read", dtype="f16", store="int8", batch=1, new_lo=768, new_hi=768, len_lo=768, len_hi=768,
             heads=2, dim=64, page=16, kept=0.0, sizes=5),
        # the caches of a batch come back, to move to another server
        dict(name="read_batch", op="read", dtype="bf16", store="e4m3", batch=32, new_lo=700, new_hi=8000, len_lo=8000, len_hi=8000,
             heads=8, dim=128, page=64, kept=0.0, sizes=6),
        # one token of one session: the draft model's step, latency
        dict(name="attend_one", op="attend", dtype="bf16", store="bf16", batch=1, new_lo=1, new_hi=1, len_lo=900, len_hi=900,
             q_heads=12, heads=2, dim=128, page=16, window=0, lse=False, sizes=7),
        # the drafted blocks of 32 sessions are verified over their caches
        dict(name="attend_block", op="attend", dtype="bf16", store="bf16", batch=32, new_lo=8, new_hi=8, len_lo=300, len_hi=4096,
             q_heads=28, heads=4, dim=128, page=16, window=0, lse=False, sizes=8),
        # single tokens of a serving batch over long 8-bit caches
        dict(name="attend_step_e4m3", op="attend", dtype="bf16", store="e4m3", batch=64, new_lo=1, new_hi=1, len_lo=500, len_hi=16384,
             q_heads=32, heads=8, dim=128, page=64, window=0, lse=True, sizes=9),
        # chunks of prompts over what is cached of them (the largest case)
        dict(name="attend_prompt", op="attend", dtype="bf16", store="bf16", batch=8, new_lo=2048, new_hi=2048, len_lo=2048, len_hi=4096,
             q_heads=32, heads=8, dim=128, page=64, window=0, lse=False, sizes=10),
        # prompts and drafted blocks in one batch, 8-bit integers, 64-wide heads, a window
        dict(name="attend_mixed", op="attend", dtype="f16", store="int8", batch=24, new_lo=0, new_hi=700, len_lo=400, len_hi=6000,
             q_heads=14, heads=2, dim=64, page=32, window=1024, lse=True, sizes=11),
    ]


_MOST_FLOPS, _MOST_BYTES = 8.0e11, 6.0e8


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what, sizes = rng.random(), rng.randint(100, 10 ** 6)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if what < 0.30:
        block = _log_int(rng, 1, 16)
        c = dict(op="edit", dtype=rng.choice(["f16", "f16", "bf16", "f32"]), batch=_log_int(rng, 1, 128),
                 block_lo=rng.choice([0, 1, block]), block_hi=block, vocab=rng.choice([VOCAB, _log_int(rng, 30000, 200000)]),
                 hist_lo=1, hist_hi=_log_int(rng, 10, 20000), bias=rng.choice([0, 0, 8, 300]), mask=rng.random() < 0.5, sizes=sizes)
        c["block_lo"] = min(c["block_lo"], block)
        c["block_hi"] = max(c["block_hi"], 1)
    else:
        cache = dict(store=rng.choice([dtype, "e4m3", "int8"]), batch=_log_int(rng, 1, 64),
                     dim=rng.choice([64, 128, 128]), page=rng.choice([16, 16, 32, 64, 128]), sizes=sizes)
        if what < 0.45:
            kept = rng.choice([0.0, 0.1, 0.25])
            new = _log_int(rng, 200, 4096) if kept else _log_int(rng, 1, 512)
            c = dict(op="write", dtype=dtype, new_lo=rng.choice([max(1, new // 3), new]), new_hi=new, len_lo=0,
                     len_hi=0 if kept else _log_int(rng, 1, 8192), heads=rng.choice([1, 2, 4, 8]), kept=kept, **cache)
        elif what < 0.55:
            new = _log_int(rng, 30, 8192)
            c = dict(op="read", dtype=dtype, new_lo=rng.choice([1, new]), new_hi=new, len_lo=new, len_hi=rng.choice([new, new + 77]),
                     heads=rng.choice([1, 2, 4, 8]), kept=0.0, **cache)
        else:
            new = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 17, 2048)])
            q_heads, heads = rng.choice([(12, 2), (14, 2), (16, 8), (16, 16), (28, 4), (32, 8), (8, 1)])
            c = dict(op="attend", dtype=dtype, new_lo=rng.choice([min(1, new), new]), new_hi=new, len_lo=1,
                     len_hi=_log_int(rng, 64, 16384), q_heads=q_heads, heads=heads, window=rng.choice([0, 0, 0, 500]),
                     lse=rng.random() < 0.5, **cache)
            c["len_hi"] = max(c["len_hi"], new)
    while True:
        w = work(c)
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and _plain_bytes(c) <= 2.5e10:
            return c
        c["batch"] = max(1, c["batch"] * 2 // 3)
        if c["batch"] == 1 and "len_hi" in c:
            c["len_hi"] = max(c["new_hi"], c["len_hi"] * 2 // 3)


def _plain_bytes(case):
    """What the padded plain form of an attention holds at most."""
    if case["op"] != "attend":
        return 0
    long = max(case["len_hi"], case["new_hi"])
    return case["batch"] * long * 4 * (2 * case["heads"] * case["dim"] + 3 * case["q_heads"] * max(1, case["new_hi"]))


def _spread(r, lo, hi):
    """Sizes of a ragged batch: spread over their logarithm, like lengths in use."""
    return lo if lo == hi else min(hi, max(lo, int(math.exp(r.uniform(math.log(max(lo, 1)), math.log(hi + 1))))))


def _tokens(case):
    """(new tokens, tokens in the cache after them, source rows) of each request."""
    r = random.Random(case["sizes"])
    new, length, source = [], [], []
    for _ in range(case["batch"]):
        n = r.randint(case["new_lo"], case["new_hi"])
        s = n
        if case.get("kept"):
            n = max(1, math.ceil(case["kept"] * n - 1e-6))
        new.append(n)
        source.append(s)
        length.append(max(n, _spread(r, case["len_lo"], case["len_hi"])))
    return new, length, source


def _blocks(case):
    """(rows, history tokens, prompt tokens among them) of each request."""
    r = random.Random(case["sizes"])
    rows = [r.randint(case["block_lo"], case["block_hi"]) for _ in range(case["batch"])]
    rows[0] = max(rows[0], 1)
    hist = [_spread(r, case["hist_lo"], case["hist_hi"]) for _ in range(case["batch"])]
    return rows, hist, [r.randint(0, h) for h in hist]


def _prefix(counts, dev):
    return torch.tensor([0] + counts).cumsum(0).to(torch.int32).to(dev)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if case["op"] == "edit":
        rows, hist, prompt = _blocks(case)
        n, vocab, batch = sum(rows), case["vocab"], case["batch"]
        ld = -(-vocab // 8) * 8
        # tokens of a text: a few are frequent
        common = (torch.rand(sum(hist) + n, generator=g, device=dev) ** 4 * vocab).int().clamp_(max=vocab - 1)
        z = (2.5 * normal(n, ld)).to(DTYPES[case["dtype"]])
        s = dict(op="edit", z=z, vocab=vocab, row_offsets=_prefix(rows, dev), history=common[:sum(hist)].contiguous(),
                 history_offsets=_prefix(hist, dev), prompt_lengths=torch.tensor(prompt, dtype=torch.int32, device=dev),
                 drafted=common[sum(hist):].contiguous(), repetition=1 + 0.3 * torch.rand(batch, generator=g, device=dev),
                 presence=torch.rand(batch, generator=g, device=dev), frequency=0.5 * torch.rand(batch, generator=g, device=dev),
                 bias_ids=None, bias_values=None, bias_offsets=None, mask=None)
        if case["bias"]:
            ids = torch.rand(batch, vocab, generator=g, device=dev).topk(case["bias"], dim=1).indices
            s.update(bias_ids=ids.int().reshape(-1).contiguous(), bias_values=3 * normal(batch * case["bias"]),
                     bias_offsets=_prefix([case["bias"]] * batch, dev))
        if case["mask"]:
            # a grammar allows few tokens in most states and nearly all inside a text
            words = -(-vocab // 32)
            few = torch.randint(-2 ** 31, 2 ** 31, (n, words), generator=g, device=dev)
            for _ in range(4):
                few &= torch.randint(-2 ** 31, 2 ** 31, (n, words), generator=g, device=dev)
            free = torch.rand(n, 1, generator=g, device=dev) < 0.3
            s["mask"] = torch.where(free, ~few, few).int().contiguous()
        return s

    new, length, source = _tokens(case)
    batch, page, heads, dim, store = case["batch"], case["page"], case["heads"], case["dim"], case["store"]
    width = max(-(-v // page) for v in length)
    used = [-(-v // page) for v in length]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=g, device=dev).int().cpu()
    table, at = torch.full((batch, width), -1, dtype=torch.int32), 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    s = dict(op=case["op"], dtype=DTYPES[case["dtype"]], store=store, table=table.to(dev), offsets=_prefix(new, dev),
             lengths=torch.tensor(length, dtype=torch.int32, device=dev), new=max(new), n=sum(new),
             k_scale=None, v_scale=None)
    # keys have channels of their own size, tokens lengths of their own; the pool holds what earlier requests left
    channel = torch.exp(0.5 * normal(heads, 1, dim))
    for name in ("k", "v"):
        x = normal(pages, heads, page, dim) * torch.exp(0.3 * normal(pages, heads, page, 1))
        if name == "k":
            x *= channel
        if store in LARGEST:
            scale = (x.abs().amax(-1) / LARGEST[store]).clamp_(min=LEAST_SCALE)
            x = x / scale[..., None]
            s[name + "_scale"] = scale
            x = x.round().clamp_(-127, 127) if store == "int8" else x.clamp_(-448, 448)
        s[name] = x.to(DTYPES[store])
        del x
    if case["op"] == "write":
        rows = sum(source) if case["kept"] else sum(new)
        # keys and values are columns of one projection
        qkv = normal(rows, 3, heads, dim) * torch.exp(0.3 * normal(rows, 1, 1, 1))
        qkv = qkv.to(s["dtype"])
        s.update(new_k=qkv[:, 1], new_v=qkv[:, 2], rows=None, row_offsets=None)
        if case["kept"]:
            key = torch.rand(rows, generator=g, device=dev).cpu()
            keep, at = [], 0
            for n, m in zip(new, source):
                keep.append(key[at:at + m].topk(n).indices.sort().values)
                at += m
            s.update(rows=torch.cat(keep).int().to(dev), row_offsets=_prefix(source, dev))
    if case["op"] == "attend":
        q_heads = case["q_heads"]
        s.update(q=(normal(sum(new), q_heads, dim) * torch.exp(0.3 * normal(1, q_heads, 1))).to(s["dtype"]),
                 scale=1 / math.sqrt(dim), window=case["window"], lse=case["lse"])
    if own:
        from paper_2605_02218_b200 import api
        s["cache"] = api.PagedCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    return s


# ---- the calls ----------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _call(state)
    return {"edit": _plain_edit, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[state["op"]](state)


def _call(s):
    if s["op"] == "edit":
        from paper_2605_02218_b200 import api
        return api.edit_logits(s["z"], s["row_offsets"], history=s["history"], history_offsets=s["history_offsets"],
                               prompt_lengths=s["prompt_lengths"], drafted=s["drafted"], repetition=s["repetition"],
                               presence=s["presence"], frequency=s["frequency"], bias_ids=s["bias_ids"],
                               bias_values=s["bias_values"], bias_offsets=s["bias_offsets"], mask=s["mask"],
                               vocab=s["vocab"])[:, :s["vocab"]]
    cache, tokens = s["cache"], (s["offsets"], s["lengths"], s["table"])
    if s["op"] == "write":
        cache.write(s["new_k"], s["new_v"], *tokens, rows=s["rows"], row_offsets=s["row_offsets"])
        return _cache(s)
    if s["op"] == "read":
        return cache.read(*tokens, s["n"], dtype=s["dtype"])
    return cache.attend(s["q"], *tokens, scale=s["scale"], window=s["window"], max_new=s["new"], lse=s["lse"])


def _cache(s):
    return [s[name] for name in ("k", "v", "k_scale", "v_scale") if s[name] is not None]


# ---- plain forms --------------------------------------------------------------------------------------------------------

def _plain_edit(s):
    z, vocab = s["z"], s["vocab"]
    n, batch, dev = z.shape[0], s["row_offsets"].numel() - 1, z.device
    request = torch.searchsorted(s["row_offsets"], torch.arange(n, device=dev, dtype=torch.int32), right=True) - 1
    # how often each request's history has a token at all, and after the prompt
    i = torch.arange(s["history"].numel(), device=dev, dtype=torch.int32)
    of = torch.searchsorted(s["history_offsets"], i, right=True) - 1
    flat = of * vocab + s["history"]
    answered = (i - s["history_offsets"][of] >= s["prompt_lengths"][of]).int()
    seen = torch.zeros(batch * vocab, dtype=torch.int32, device=dev).scatter_add_(0, flat, torch.ones_like(answered)).view(batch, vocab)
    times = torch.zeros(batch * vocab, dtype=torch.int32, device=dev).scatter_add_(0, flat, answered).view(batch, vocab)
    # the drafted tokens before a row count for it
    row = torch.arange(n, device=dev)
    before = ((request[:, None] == request) & (row[:, None] > row)).int()
    block = torch.zeros(n, vocab, dtype=torch.int32, device=dev).scatter_add_(1, s["drafted"].long().expand(n, n), before)
    times = times[request] + block
    seen = (seen[request] + block) > 0
    x = z[:, :vocab].float()
    r = s["repetition"][request, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][request, None] * times - torch.where(times > 0, s["presence"][request, None], 0.0)
    if s["bias_ids"] is not None:
        j = torch.arange(s["bias_ids"].numel(), device=dev, dtype=torch.int32)
        of = torch.searchsorted(s["bias_offsets"], j, right=True) - 1
        x = x + torch.zeros(batch, vocab, device=dev).index_put_((of, s["bias_ids"].long()), s["bias_values"])[request]
    if s["mask"] is not None:
        w = torch.arange(vocab, device=dev)
        x = x.masked_fill((s["mask"][:, w // 32] >> (w % 32).int()) & 1 == 0, -math.inf)
    return x.to(z.dtype)


def _slots(s):
    """Page and place in it of every new token."""
    i = torch.arange(s["n"], device=s["table"].device, dtype=torch.int32)
    of = torch.searchsorted(s["offsets"], i, right=True) - 1
    pos = s["lengths"][of] - s["offsets"][of + 1] + i
    page = s["k"].shape[2]
    return s["table"][of, (pos // page).long()].long(), (pos % page).long(), of


def _plain_write(s):
    page, place, of = _slots(s)
    k, v, store = s["new_k"], s["new_v"], s["store"]
    if s["rows"] is not None:
        source = s["row_offsets"][of] + s["rows"]
        k, v = k[source], v[source]
    _plain_store(s["k"], s["k_scale"], k, store, page, place)
    _plain_store(s["v"], s["v_scale"], v, store, page, place)
    return _cache(s)


def _plain_store(cache, scales, x, store, page, place):
    if store not in LARGEST:
        cache[page, :, place] = x.to(cache.dtype)
        return
    most = torch.full((), LARGEST[store], device=x.device)    # a divisor on the host would become a product with its inverse
    scale = (x.float().abs().amax(-1) / most).clamp(min=LEAST_SCALE)
    t = x.double() / scale.double()[..., None]                # 64 bits: quotients next to a border round the right way
    if store == "int8":
        t = t.round().clamp(-127, 127)
    else:
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        t = ((t / step).round() * step).clamp(-448, 448)
    cache[page, :, place] = t.to(cache.dtype)
    scales[page, :, place] = scale


def _plain_read(s):
    page, place, _ = _slots(s)
    got = []
    for x, scale in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])):
        x = x[page, :, place].float()
        got.append((x if scale is None else x * scale[page, :, place][..., None]).to(s["dtype"]))
    return got


def _plain_attend(s):
    q, table, lengths, offsets, dev = s["q"], s["table"], s["lengths"], s["offsets"], s["q"].device
    batch, new = lengths.numel(), max(s["new"], 1)
    n, q_heads, dim = q.shape
    heads, page = s["k"].shape[1], s["k"].shape[2]
    long = table.shape[1] * page
    at = torch.arange(long, device=dev)
    filled = at < lengths[:, None]

    def dense(x, scale):
        pages = table.long().clamp(min=0)
        y = x[pages].float()
        if scale is not None:
            y = y * scale[pages][..., None]
        y = y.permute(0, 2, 1, 3, 4).reshape(batch, heads, long, dim)
        return torch.where(filled[:, None, :, None], y, 0.0)

    i = torch.arange(new, device=dev)
    rows = (offsets[:-1, None] + i).clamp(max=n - 1)
    count = offsets[1:] - offsets[:-1]
    pos = (lengths - count)[:, None] + i
    x = q[rows].float().reshape(batch, new, heads, q_heads // heads, dim).permute(0, 2, 3, 1, 4)
    x = x.reshape(batch, heads, -1, dim) @ dense(s["k"], s["k_scale"]).transpose(2, 3) * s["scale"]
    see = (at <= pos[:, :, None]) & filled[:, None]
    if s["window"]:
        see &= at > pos[:, :, None] - s["window"]
    x = x.view(batch, heads, q_heads // heads, new, long).masked_fill_(~see[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = x.view(batch, heads, -1, long) @ dense(s["v"], s["v_scale"])
    o = o.view(batch, heads, -1, new, dim) / torch.where(total == 0, 1.0, total)
    token = torch.arange(n, device=dev, dtype=torch.int32)
    of = torch.searchsorted(offsets, token, right=True) - 1
    mine = (token - offsets[of]).long()
    out = o.permute(0, 3, 1, 2, 4)[of, mine].reshape(n, q_heads, dim).to(q.dtype)
    if not s["lse"]:
        return out
    lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2)[of, mine].reshape(n, q_heads)
    return out, lse


# ---- the definitions in 64 bits, request by request ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"edit": _exact_edit, "write": _exact_write, "read": _exact_read, "attend": _exact_attend}[case["op"]](s)


def _exact_edit(s):
    vocab, off, hist_off = s["vocab"], s["row_offsets"].tolist(), s["history_offsets"].tolist()
    out = torch.empty(s["z"].shape[0], vocab, dtype=torch.float64, device=s["z"].device)
    bit = torch.arange(32, device=out.device)
    for b in range(len(off) - 1):
        past = s["history"][hist_off[b]:hist_off[b + 1]].long()
        answer = past[int(s["prompt_lengths"][b]):]
        r, a, f = (float(s[name][b]) for name in ("repetition", "presence", "frequency"))
        for row in range(off[b], off[b + 1]):
            drafted = s["drafted"][off[b]:row].long()
            x = s["z"][row, :vocab].double()
            for token in (torch.unique(torch.cat([past, drafted])),):
                x[token] = torch.where(x[token] > 0, x[token] / r, x[token] * r)
            token, c = torch.unique(torch.cat([answer, drafted]), return_counts=True)
            x[token] -= f * c.double() + a
            if s["bias_ids"] is not None:
                lo, hi = int(s["bias_offsets"][b]), int(s["bias_offsets"][b + 1])
                x[s["bias_ids"][lo:hi].long()] += s["bias_values"][lo:hi].double()
            if s["mask"] is not None:
                allowed = ((s["mask"][row].long()[:, None] >> bit) & 1).reshape(-1)[:vocab] == 1
                x[~allowed] = -math.inf
            out[row] = x
    return out


def _exact_rows(s, b):
    """Pages and places of the positions of request b that its new tokens have."""
    lo, hi, length, page = int(s["offsets"][b]), int(s["offsets"][b + 1]), int(s["lengths"][b]), s["k"].shape[2]
    pos = torch.arange(length - (hi - lo), length, device=s["k"].device)
    return lo, hi, s["table"][b].long()[pos // page], pos % page


def _exact_write(s):
    out = [s[name].double() for name in ("k", "v", "k_scale", "v_scale") if s[name] is not None]
    for b in range(s["lengths"].numel()):
        lo, hi, page, place = _exact_rows(s, b)
        for k, name in enumerate(("new_k", "new_v")):
            x = s[name]
            x = x[lo:hi] if s["rows"] is None else x[s["rows"][lo:hi].long() + int(s["row_offsets"][b])]
            x = x.double()
            if s["store"] not in LARGEST:
                out[k][page, :, place] = x.to(DTYPES[s["store"]]).double()
                continue
            most = LARGEST[s["store"]]
            scale = (x.abs().amax(-1) / most).clamp(min=LEAST_SCALE)
            x = x / scale.float().double()[..., None]         # the cache keeps the scale in 32 bits
            if s["store"] == "e4m3":
                mantissa, exponent = torch.frexp(x)
                unit = torch.ldexp(torch.ones_like(x), exponent.clamp(min=-5) - 4)   # four bits, from 2^-6 down a fixed step
                x = torch.round(x / unit) * unit
            else:
                x = torch.round(x)
            out[k][page, :, place] = x.clamp(-most, most)
            out[2 + k][page, :, place] = scale
    return out


def _exact_read(s):
    got = []
    for name in ("k", "v"):
        part = []
        for b in range(s["lengths"].numel()):
            _, _, page, place = _exact_rows(s, b)
            x = s[name][page, :, place].double()
            part.append(x if s[name + "_scale"] is None else x * s[name + "_scale"][page, :, place].double()[..., None])
        got.append(torch.cat(part))
    return got


def _exact_attend(s):
    q, page = s["q"], s["k"].shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    group = q.shape[1] // s["k"].shape[1]
    for b in range(s["lengths"].numel()):
        lo, hi, length = int(s["offsets"][b]), int(s["offsets"][b + 1]), int(s["lengths"][b])
        if lo == hi or not length:
            continue
        pos = torch.arange(length, device=q.device)
        at = s["table"][b].long()[pos // page], pos % page
        mine = torch.arange(length - (hi - lo), length, device=q.device)[:, None]
        hidden = pos > mine
        if s["window"]:
            hidden |= pos <= mine - s["window"]
        for h in range(q.shape[1]):
            k, v = (s[name][at[0], h // group, at[1]].double() for name in ("k", "v"))
            if s["k_scale"] is not None:
                k *= s["k_scale"][at[0], h // group, at[1]].double()[:, None]
                v *= s["v_scale"][at[0], h // group, at[1]].double()[:, None]
            x = (q[lo:hi, h].double() @ k.T * s["scale"]).masked_fill(hidden, -math.inf)
            lse[lo:hi, h] = torch.logsumexp(x, -1)
            out[lo:hi, h] = torch.softmax(x, -1).nan_to_num() @ v
    return (out, lse) if s["lse"] else out


# ---- floors -------------------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "edit":
        rows, hist, _ = _blocks(case)
        n, e = sum(rows), BYTES[case["dtype"]]
        size = 2.0 * n * case["vocab"] * e + 4 * (sum(hist) + n) + 8 * case["bias"] * case["batch"]
        return {"bytes": size + (n * 4.0 * -(-case["vocab"] // 32) if case["mask"] else 0), "flops": float(n) * case["vocab"]}
    new, length, _ = _tokens(case)
    row = case["heads"] * (case["dim"] * BYTES[case["store"]] + (4 if case["store"] in LARGEST else 0))
    n, e = float(sum(new)), BYTES[case["dtype"]]
    if case["op"] != "attend":
        return {"bytes": 2 * n * (row + case["heads"] * case["dim"] * e), "flops": 4 * n * case["heads"] * case["dim"]}
    w = case["window"] or 1 << 40
    seen = sum(min(v, m + w - 1) if m else 0 for m, v in zip(new, length))          # keys that some row attends to
    pairs = sum(min(v - m + i + 1, w) for m, v in zip(new, length) for i in range(m))
    size = 2.0 * seen * row + 2 * n * case["q_heads"] * case["dim"] * e + (4 * n * case["q_heads"] if case["lse"] else 0)
    return {"bytes": size, "flops": 4.0 * pairs * case["q_heads"] * case["dim"]}
