"""Attention over a cache of secret shares: timed cases of one party's local work.

Every number is a word of the ring Z_{2^64} (int64 tensors hold its bits) and every output has to be
exact.  The operators, for party i (0 or 1), with t(x) the share-local rescaling by 2^f
(party 0: floor(x / 2^f) on the signed word; party 1: -floor(-x / 2^f)):

``cache_write``  the exchanged masked rows of new tokens are opened into the cache:
                 F[slot] = D_0 + D_1,  X_i[slot] = B_i + i F[slot]  (X_0 + X_1 is the cached value).
``cache_read``   rows of the cache as operands of a share product: E = F[slot], A_i = X_i[slot] - i F[slot].
``rotate``       rescaling of a projection, position rotation and masking of the result, in one pass.
``scores``       queries times cached keys: t(C_i + E X_i^T + A_i F^T) - M_i for the keys a row sees.
``weights``      the opened masked scores squared, (s + c)^2, masked again, with the sum of every row.
``values``       weights times cached values: t(C_i + E X_i + A_i F) - M_i.

Masked values, shares and triple parts are uniform over the ring whatever the secrets are, so all of
them are drawn as uniform words; tables of the rotation, lengths and pages are as a server has them.
"""
from __future__ import annotations

import math

import torch

own = False

# Two products per party (E X and A F) and, per 64-bit multiply-add, 36 products of signed base-256
# digits of two operations each: the fewest exact int8 operations a word product takes.
INT8_OPS_PER_MAC = 72

FRAC = 16                         # fractional bits of the fixed-point encoding
BIAS = 5 << FRAC                  # c of the weights (s + c)^2


def listed():
    one = dict(new=1, head_mask=0)
    return [
        # keys of a batch of prompts of LLaMA-2-13B (40 heads of 128) on their way into the cache
        dict(name="write_prompt", op="cache_write", tokens=2048, width=5120, page=64, party=1),
        # latent rows (512 and a rotated part of 64) of one long sequence, to be expanded to keys and values
        dict(name="read_latent", op="cache_read", tokens=6000, width=576, page=16, party=1),
        # the new token of one LLaMA-7B request: a handful of microseconds, launch and host time
        dict(name="rotate_one_token", op="rotate", tokens=1, heads=32, dim=128, rot=128, interleaved=0, masked=1, fused=1,
             party=0),
        # queries of a LLaMA-2-13B prompt batch out of the fused projection's result
        dict(name="rotate_prompt", op="rotate", tokens=2048, heads=40, dim=128, rot=128, interleaved=0, masked=1, fused=3,
             party=1),
        # sixteen requests, one new token each, four query heads per key head, up to 8192 cached tokens
        dict(one, name="scores_decode", op="scores", seqs=16, cached=8192, ragged=1, heads=32, kv_heads=8, dim=128, row=128,
             page=64, party=1),
        # four LLaMA-7B prompts of up to 512 tokens (the paper's input length)
        dict(name="scores_prompt", op="scores", seqs=4, new=512, cached=0, ragged=1, heads=32, kv_heads=32, dim=128, row=128,
             page=64, party=1, head_mask=0),
        # latent attention, absorbed form: 64 query heads over one row of 512 + 64 words a token
        dict(one, name="scores_latent", op="scores", seqs=4, cached=4000, ragged=1, heads=64, kv_heads=1, dim=576, row=576,
             page=16, party=0),
        # the squared scores of the decoding batch and of the prompts above
        dict(one, name="weights_decode", op="weights", seqs=16, cached=8192, ragged=1, heads=32, kv_heads=8, page=64, party=1),
        dict(name="weights_prompt", op="weights", seqs=4, new=512, cached=0, ragged=1, heads=32, kv_heads=32, page=64, party=0,
             head_mask=0),
        # one OPT-125m request in the middle of its answer, half of the heads inactive
        dict(name="values_opt_token", op="values", seqs=1, new=1, cached=200, ragged=0, heads=12, kv_heads=12, dim=64, row=64,
             page=16, party=1, head_mask=1),
        # the decoding batch over its cached values
        dict(one, name="values_decode", op="values", seqs=16, cached=8192, ragged=1, heads=32, kv_heads=8, dim=128, row=128,
             page=64, party=0),
        # a chunk of 512 tokens of a long prompt behind 4096 cached ones
        dict(name="values_chunk", op="values", seqs=1, new=512, cached=4096, ragged=0, heads=32, kv_heads=8, dim=128, row=128,
             page=64, party=1, head_mask=0),
    ]


# ---------------------------------------------------------------------------
# further cases of the same ranges
# ---------------------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rows(rng, op):
    return dict(op=op, tokens=_log(rng, 1, 8192), width=2 * _log(rng, 32, 2560), page=16 * _log(rng, 1, 16),
                party=rng.randint(0, 1))


def _draw_rotate(rng):
    dim = rng.choice((64, 80, 96, 128, 128, 192, 576))
    rot = rng.choice((dim, dim, 64, 2 * rng.randint(1, dim // 2)))
    return dict(op="rotate", tokens=_log(rng, 1, 4096), heads=rng.randint(1, 64), dim=dim, rot=rot,
                interleaved=rng.randint(0, 1), masked=rng.randint(0, 1), fused=rng.choice((1, 2, 3)), party=rng.randint(0, 1))


def _draw_attention(rng, op):
    kind = rng.choice(("decode", "decode", "prompt", "chunk", "latent"))
    c = dict(op=op, ragged=rng.randint(0, 1), page=16 * _log(rng, 1, 16), party=rng.randint(0, 1),
             head_mask=rng.choice((0, 0, 1)))
    if kind == "latent":
        heads = rng.randint(8, 128)
        c.update(seqs=_log(rng, 1, 8), new=rng.choice((1, 1, 2, 37)), cached=_log(rng, 16, 8192), heads=heads, kv_heads=1)
        row = 2 * rng.randint(64, 288)
        dim = row if op == "scores" else 2 * rng.randint(32, row // 2)
    else:
        kv = rng.choice((1, 2, 4, 8, 12, 32))
        c.update(kv_heads=kv, heads=kv * rng.choice((1, 1, 4, 7, 8)) if kv <= 8 else kv)
        row = dim = rng.choice((64, 64, 80, 96, 128, 128, 192, 2 * rng.randint(8, 128)))
        if kind == "decode":
            c.update(seqs=_log(rng, 1, 32), new=1, cached=_log(rng, 1, 16384))
        elif kind == "prompt":
            c.update(seqs=rng.randint(1, 4), new=_log(rng, 2, 1024), cached=0)
        else:
            c.update(seqs=rng.randint(1, 2), new=_log(rng, 2, 512), cached=_log(rng, 16, 8192))
    if op != "weights":
        c.update(dim=dim, row=row)
    return c


def draw(rng):
    largest = max(_seconds(c) for c in listed())
    while True:
        op = rng.choice(("cache_write", "cache_read", "rotate", "scores", "scores", "weights", "values", "values"))
        if op in ("cache_write", "cache_read"):
            c = _draw_rows(rng, op)
        elif op == "rotate":
            c = _draw_rotate(rng)
        else:
            c = _draw_attention(rng, op)
        if _seconds(c) <= largest and _state_words(c) < 4e8:
            return c


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, cached tokens in all) of every sequence; ragged batches run down from the longest to a third of it."""
    out = []
    for s in range(case["seqs"]):
        share = 1.0 - (s / case["seqs"]) * 0.67 if case["ragged"] else 1.0
        new = max(1, int(case["new"] * share))
        out.append((new, int(case["cached"] * share) + new))
    return out


def _ld(case):
    """Words in a row of a score matrix: the longest sequence, rounded up to a whole page."""
    longest = max(n for _, n in _lengths(case))
    return -(-longest // case["page"]) * case["page"]


def _visible(case):
    """Keys that all rows of one head see together."""
    return sum(sum(kv - new + j + 1 for j in range(new)) for new, kv in _lengths(case))


def work(case):
    op = case["op"]
    if op in ("cache_write", "cache_read"):
        n = case["tokens"] * case["width"]
        return {"bytes": (40 if op == "cache_write" else 32) * n, "flops": 0}
    if op == "rotate":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": (24 if case["masked"] else 16) * n, "flops": 0}
    lens, heads = _lengths(case), case["heads"]
    active = heads / 2 if case["head_mask"] else heads
    seen = _visible(case) * active
    rows = sum(new for new, _ in lens) * heads
    if op == "weights":
        return {"bytes": 48 * seen + 8 * rows, "flops": 0}
    pool = sum(kv for _, kv in lens) * case["kv_heads"] * case["dim"]
    macs = 2 * seen * case["dim"]
    if op == "scores":
        moved = 16 * pool + 16 * rows * case["dim"] + 24 * seen
    else:
        moved = 16 * pool + 16 * seen + 24 * rows * case["dim"]
    return {"bytes": moved, "flops": INT8_OPS_PER_MAC * macs}


def _seconds(case):
    """A rough cost, to compare cases by."""
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 2.5e15)


def _state_words(case):
    if case["op"] in ("cache_write", "cache_read"):
        return 8 * case["tokens"] * case["width"]
    if case["op"] == "rotate":
        return 6 * case["tokens"] * case["heads"] * case["dim"]
    lens = _lengths(case)
    table = sum(new for new, _ in lens) * case["heads"] * _ld(case)
    padded = len(lens) * max(new for new, _ in lens) * case["heads"] * _ld(case)
    return 5 * table + padded + 4 * len(lens) * _ld(case) * case["kv_heads"] * case.get("row", 0)


# ---------------------------------------------------------------------------
# states
# ---------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _words(gen, *shape):
    return torch.randint(-2 ** 63, 2 ** 63 - 1, shape, dtype=torch.int64, device="cuda", generator=gen)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_rows(case, gen):
    t, w, page = case["tokens"], case["width"], case["page"]
    pages = -(-t // page) + 3
    order = torch.randperm(pages, device="cuda", generator=gen)
    at = torch.arange(t, device="cuda")
    slots = (order[at // page] * page + at % page).to(torch.int32)
    s = dict(slots=slots, f_pool=_words(gen, pages * page, w), x_pool=_words(gen, pages * page, w))
    if case["op"] == "cache_write":
        s.update(d_0=_words(gen, t, w), d_1=_words(gen, t, w), b_i=_words(gen, t, w))
    else:
        s.update(e=torch.empty(t, w, dtype=torch.int64, device="cuda"), a_i=torch.empty(t, w, dtype=torch.int64, device="cuda"))
    return s


def _prepare_rotate(case, gen):
    t, h, d, rot = case["tokens"], case["heads"], case["dim"], case["rot"]
    longest = 4096
    angle = torch.arange(longest, dtype=torch.float64)[:, None] * \
        10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    fixed = lambda x: torch.round(x * 2 ** FRAC).to(torch.int64).cuda()
    # the heads to rotate are a column range of the (fused) projection's result
    wide = _words(gen, t, case["fused"] * h * d)
    return dict(x_i=wide[:, :h * d], positions=torch.randint(0, longest, (t,), device="cuda", generator=gen).to(torch.int32),
                cos=fixed(torch.cos(angle)), sin=fixed(torch.sin(angle)),
                m_i=_words(gen, t, h * d) if case["masked"] else None,
                out=torch.empty(t, h * d, dtype=torch.int64, device="cuda"))


def _prepare_attention(case, gen):
    lens, page, heads, kvh = _lengths(case), case["page"], case["heads"], case["kv_heads"]
    ld, n_seq = _ld(case), len(lens)
    t = sum(new for new, _ in lens)
    each = [-(-kv // page) for _, kv in lens]
    pages = sum(each) + 2
    order = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros(n_seq, ld // page, dtype=torch.int32, device="cuda")
    first = 0
    for s, n in enumerate(each):
        table[s, :n] = order[first:first + n]
        first += n
    starts = [0]
    for new, _ in lens:
        starts.append(starts[-1] + new)
    mask = None
    if case["head_mask"]:
        # half of the heads of every token are active
        rank = torch.rand(t, heads, device="cuda", generator=gen).argsort(1).argsort(1)
        mask = (rank < heads // 2).to(torch.uint8)
    s = dict(q_start=_int32(starts), kv_len=_int32([kv for _, kv in lens]), table=table, head_mask=mask, t=t, ld=ld,
             max_new=max(new for new, _ in lens))
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.int64, device="cuda")
    if case["op"] == "weights":
        s.update(d_0=_words(gen, t, heads, ld), d_1=_words(gen, t, heads, ld), r_i=_words(gen, t, heads, ld),
                 r2_i=_words(gen, t, heads, ld), m_i=_words(gen, t, heads, ld), out=zeros(t, heads, ld), sums=zeros(t, heads))
    else:
        d = case["dim"]
        pool = (pages, page, kvh, case["row"])
        s.update(f_pool=_words(gen, *pool), x_pool=_words(gen, *pool))
        left, right = ((t, heads, d), (t, heads, ld)) if case["op"] == "scores" else ((t, heads, ld), (t, heads, d))
        s.update(e=_words(gen, *left), a_i=_words(gen, *left), c_i=_words(gen, *right), m_i=_words(gen, *right),
                 out=zeros(*right))
    return s


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    if op in ("cache_write", "cache_read"):
        s = _prepare_rows(case, gen)
    elif op == "rotate":
        s = _prepare_rotate(case, gen)
    else:
        s = _prepare_attention(case, gen)
    s["case"] = case
    if own:
        import paper_2505_07239_amd as comet
        s["ctx"] = comet.Context(0)
        if "q_start" in s:
            s["batch"] = comet.KVBatch(s["t"], case["heads"], case["kv_heads"], s["q_start"], s["kv_len"], s["table"],
                                       case["page"], s["max_new"], head_mask=s["head_mask"])
    return s


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------

def _rescale(x, party, bits):
    return x >> bits if party == 0 else -((-x) >> bits)


def _product(a, b):
    """a @ b mod 2^64 in limbs of 16 bits: their products and sums stay below 2^53, where float64 is exact."""
    left = [((a >> (16 * i)) & 0xFFFF).to(torch.float64) for i in range(4)]
    right = [((b >> (16 * i)) & 0xFFFF).to(torch.float64) for i in range(4)]
    total = None
    for i in range(4):
        for j in range(4 - i):
            term = torch.matmul(left[i], right[j]).to(torch.int64) << (16 * (i + j))
            total = term if total is None else total + term
    return total


def _layout(s):
    """Rows of the padded batch: token of every (sequence, place), and how many keys each of its heads sees."""
    case, q, kv = s["case"], s["q_start"].long(), s["kv_len"].long()
    new = q[1:] - q[:-1]
    place = torch.arange(s["max_new"], device=q.device)
    live = place[None, :] < new[:, None]
    token = torch.where(live, q[:-1, None] + place[None, :], 0)
    seen = (kv[:, None] - new[:, None] + place[None, :] + 1).clamp(min=0)
    seen = torch.where(live, seen, 0)[:, :, None].expand(-1, -1, case["heads"])
    if s["head_mask"] is not None:
        seen = seen * s["head_mask"][token].long()
    return token, live, seen


def _pad(x, token, kvh):
    """[tokens, heads, w] -> [sequence, key head, place x group, w]."""
    n_seq, places = token.shape
    heads, w = x.shape[1:]
    x = x[token].view(n_seq, places, kvh, heads // kvh, w).transpose(1, 2)
    return x.reshape(n_seq, kvh, places * (heads // kvh), w)


def _unpad(x, places, heads):
    """The other way: [sequence, key head, place x group, w] -> [sequence, place, head, w]."""
    n_seq, kvh, _, w = x.shape
    return x.view(n_seq, kvh, places, heads // kvh, w).transpose(1, 2).reshape(n_seq, places, heads, w)


def _cached(pool, s, d):
    """[sequence, key head, cached token, d] out of the pages."""
    rows = pool[s["table"].long()].flatten(1, 2)[:, :, :, :d]
    return rows.transpose(1, 2)


def _run_plain(s):
    case = s["case"]
    op, party = case["op"], case["party"]
    if op == "cache_write":
        f = s["d_0"] + s["d_1"]
        at = s["slots"].long()
        s["f_pool"][at] = f
        s["x_pool"][at] = s["b_i"] + party * f
        return s["f_pool"], s["x_pool"]
    if op == "cache_read":
        at = s["slots"].long()
        e = s["f_pool"][at]
        return e, s["x_pool"][at] - party * e
    if op == "rotate":
        t, h, d, half = case["tokens"], case["heads"], case["dim"], case["rot"] // 2
        x = _rescale(s["x_i"], party, FRAC).view(t, h, d)
        at = s["positions"].long()
        c, n = s["cos"][at][:, None, :], s["sin"][at][:, None, :]
        if case["interleaved"]:
            x1, x2 = x[:, :, 0:2 * half:2], x[:, :, 1:2 * half:2]
        else:
            x1, x2 = x[:, :, :half], x[:, :, half:2 * half]
        y1, y2 = _rescale(x1 * c - x2 * n, party, FRAC), _rescale(x2 * c + x1 * n, party, FRAC)
        turned = torch.stack((y1, y2), -1).flatten(2) if case["interleaved"] else torch.cat((y1, y2), -1)
        y = torch.cat((turned, x[:, :, 2 * half:]), -1).view(t, h * d)
        return y if s["m_i"] is None else y - s["m_i"]
    token, live, seen = _layout(s)
    heads, places = case["heads"], s["max_new"]
    keys = torch.arange(s["ld"], device="cuda")
    if op == "weights":
        u = s["d_0"] + s["d_1"] + BIAS
        w = _rescale(party * u * u + 2 * u * s["r_i"] + s["r2_i"], party, FRAC)
        count = torch.zeros(s["t"], heads, dtype=torch.int64, device="cuda")
        count[token[live]] = seen[live]
        shown = keys < count[:, :, None]
        return torch.where(shown, w - s["m_i"], 0), torch.where(shown, w, 0).sum(-1)
    kvh, d = case["kv_heads"], case["dim"]
    xs, fs = _cached(s["x_pool"], s, d), _cached(s["f_pool"], s, d)
    e, a = _pad(s["e"], token, kvh), _pad(s["a_i"], token, kvh)
    out = torch.zeros_like(s["out"])
    if op == "scores":
        z = _unpad(_product(e, xs.transpose(2, 3)) + _product(a, fs.transpose(2, 3)), places, heads)[live]
        at = token[live]
        z = _rescale(z + s["c_i"][at], party, FRAC) - s["m_i"][at]
        out[at] = torch.where(keys < seen[live][:, :, None], z, 0)
        return out
    shown = keys < _pad_counts(seen, kvh)
    z = _product(torch.where(shown, e, 0), xs) + _product(torch.where(shown, a, 0), fs)
    at = token[live]
    out[at] = _rescale(_unpad(z, places, heads)[live] + s["c_i"][at], party, FRAC) - s["m_i"][at]
    return out


def _pad_counts(seen, kvh):
    n_seq, places, heads = seen.shape
    return seen.reshape(n_seq, places, kvh, heads // kvh).transpose(1, 2).reshape(n_seq, kvh, -1, 1)


def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    op, party = case["op"], case["party"]
    if op == "cache_write":
        ctx.cache_write(party, s["d_0"], s["d_1"], s["b_i"], s["slots"], s["f_pool"], s["x_pool"])
        return s["f_pool"], s["x_pool"]
    if op == "cache_read":
        return ctx.cache_read(party, s["f_pool"], s["x_pool"], s["slots"], out=(s["e"], s["a_i"]))
    if op == "rotate":
        return ctx.rotate_share(party, s["x_i"], s["positions"], s["cos"], s["sin"], case["heads"], FRAC, FRAC, m_i=s["m_i"],
                                interleaved=bool(case["interleaved"]), out=s["out"])
    if op == "weights":
        return ctx.attention_weights(party, s["batch"], s["d_0"], s["d_1"], s["r_i"], s["r2_i"], BIAS, FRAC, m_i=s["m_i"],
                                     out=(s["out"], s["sums"]))
    call = ctx.attention_scores if op == "scores" else ctx.attention_values
    return call(party, s["batch"], s["e"], s["a_i"], s["f_pool"], s["x_pool"], s["c_i"], FRAC, m_i=s["m_i"], out=s["out"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# the definition, in 64-bit integers, one sequence and head at a time
# ---------------------------------------------------------------------------

def _dot(rows, cols):
    """rows [n, k] times cols [m, k] transposed: every product of two words, added up mod 2^64."""
    out = torch.empty(rows.shape[0], cols.shape[0], dtype=torch.int64, device=rows.device)
    step = max(1, 2 ** 27 // max(1, cols.numel()))
    for r in range(0, rows.shape[0], step):
        out[r:r + step] = (rows[r:r + step, None, :] * cols[None, :, :]).sum(-1)
    return out


def exact(case, seed):
    s = _prepared(case, seed)
    op, party = case["op"], case["party"]
    floor = lambda x: torch.div(x, 2 ** FRAC, rounding_mode="floor")
    scaled = (lambda x: floor(x)) if party == 0 else (lambda x: -floor(-x))
    if op == "cache_write":
        for i, slot in enumerate(s["slots"].tolist()):
            s["f_pool"][slot] = s["d_1"][i] + s["d_0"][i]
            s["x_pool"][slot] = s["b_i"][i] + (s["f_pool"][slot] if party else 0)
        return s["f_pool"], s["x_pool"]
    if op == "cache_read":
        rows = [(s["f_pool"][n], s["x_pool"][n]) for n in s["slots"].tolist()]
        return torch.stack([f for f, _ in rows]), torch.stack([x - f if party else x for f, x in rows])
    if op == "rotate":
        d, half = case["dim"], case["rot"] // 2
        x = scaled(s["x_i"]).reshape(-1, case["heads"], d)
        out = x.clone()
        for k in range(half):
            lo, hi = (2 * k, 2 * k + 1) if case["interleaved"] else (k, k + half)
            c, n = s["cos"][s["positions"].long(), k, None], s["sin"][s["positions"].long(), k, None]
            out[:, :, lo] = scaled(c * x[:, :, lo] - n * x[:, :, hi])
            out[:, :, hi] = scaled(n * x[:, :, lo] + c * x[:, :, hi])
        out = out.reshape(out.shape[0], -1)
        return out if s["m_i"] is None else out - s["m_i"]
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros_like(s["out"])
    sums = torch.zeros(s["t"], case["heads"], dtype=torch.int64, device="cuda")
    first = 0
    for q, (new, kv) in enumerate(_lengths(case)):
        rows = slice(first, first + new)
        first += new
        # keys at or before a token's own place, for its active heads
        shown = torch.arange(kv, device="cuda")[None, :] <= torch.arange(kv - new, kv, device="cuda")[:, None]
        slots = [int(s["table"][q, j // case["page"]]) * case["page"] + j % case["page"] for j in range(kv)]
        slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
        for h in range(case["heads"]):
            seen = shown if s["head_mask"] is None else shown & (s["head_mask"][rows, h, None] != 0)
            if op == "weights":
                r, u = s["r_i"][rows, h, :kv], s["d_1"][rows, h, :kv] + s["d_0"][rows, h, :kv] + BIAS
                w = s["r2_i"][rows, h, :kv] + u * r + u * r
                w = scaled(w + u * u if party else w)
                out[rows, h, :kv] = (w - s["m_i"][rows, h, :kv]) * seen
                sums[rows, h] = (w * seen).sum(-1)
                continue
            d = case["dim"]
            xs = s["x_pool"].flatten(0, 1)[slots, h // group, :d]
            fs = s["f_pool"].flatten(0, 1)[slots, h // group, :d]
            if op == "scores":
                z = s["c_i"][rows, h, :kv] + _dot(s["e"][rows, h], xs) + _dot(s["a_i"][rows, h], fs)
                out[rows, h, :kv] = (scaled(z) - s["m_i"][rows, h, :kv]) * seen
            else:
                z = s["c_i"][rows, h] + _dot(s["e"][rows, h, :kv] * seen, xs.t().contiguous())
                z = z + _dot(s["a_i"][rows, h, :kv] * seen, fs.t().contiguous())
                out[rows, h] = scaled(z) - s["m_i"][rows, h]
    return (out, sums) if op == "weights" else out


def _prepared(case, seed):
    """The inputs of ``prepare`` without the framework's handle."""
    gen = _generator(seed)
    make = {"cache_write": _prepare_rows, "cache_read": _prepare_rows, "rotate": _prepare_rotate}
    return make.get(case["op"], _prepare_attention)(case, gen)
