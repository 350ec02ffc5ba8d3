"""Attention over a cache of shares: calls that the documentation allows and that are easily got wrong, word for word
against the oracle or a closed form."""

import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import attention as oa                    # noqa: E402
from test_gpu_attention import PATTERN, Case, U, check_scores, check_values, ctx, down, ints, pattern, say, u64, up  # noqa: E402,F401


def test_cache_rows_of_paged_pools(ctx):
    """Without a width, a slot of pools [pages, slots, key heads, words] has the words of its key heads."""
    say("cache rows of paged pools")
    pages, page, kvh, words = 3, 16, 2, 10
    f, x = (u64(3000, 1 + i, pages, page, kvh, words) for i in (0, 1))
    flat = lambda v: v.reshape(pages * page, kvh * words)
    slots = np.array([2, 47, -1, 16, 2, 48], dtype=np.int32)
    none = np.zeros((len(slots), kvh * words), dtype=U)
    for party in (0, 1):
        want = oa.cache_read(party, flat(f), flat(x), slots, none, none)
        got = ctx.cache_read(party, up(f), up(x), up(slots))
        assert all(np.array_equal(down(g), w) for g, w in zip(got, want))
        # one key head's pools without their axis, and flat ones, as before
        for shape in ((pages * page, kvh, words), (pages * page, kvh * words)):
            got = ctx.cache_read(party, up(f.reshape(shape)), up(x.reshape(shape)), up(slots))
            assert all(np.array_equal(down(g), w) for g, w in zip(got, want))
        got = ctx.cache_read(party, up(f), up(x), up(slots), width=words)      # single key heads' rows
        want = oa.cache_read(party, f.reshape(-1, words), x.reshape(-1, words), slots, none[:, :words], none[:, :words])
        assert all(np.array_equal(down(g), w) for g, w in zip(got, want))


@pytest.mark.parametrize("shape", [(0, 8), (0, 16, 2, 4)])
def test_pools_without_slots(ctx, shape):
    """Every slot is outside pools that have none: nothing is written, and what is read stays as it was."""
    say("no slots %s" % (shape,))
    pool = torch.zeros(shape, dtype=torch.int64, device="cuda")
    rows, slots = u64(3010, 1, 2, 8), ints([0, 5])
    ctx.cache_write(1, up(rows), up(rows), up(rows), slots, pool, pool.clone())
    out = (up(pattern(2, 8)), up(pattern(2, 8)))
    ctx.cache_read(1, pool, pool, slots, out=out)
    assert all(np.array_equal(down(o), pattern(2, 8)) for o in out)
    assert not any(down(o).any() for o in ctx.cache_read(0, pool, pool, slots))


def test_numbers_beyond_32_bits_are_refused(ctx):
    """Not cut to their low 32 bits: a bound of 2^32 tokens would read as none, 2^32 + 16 as 16."""
    say("numbers beyond 32 bits")
    import paper_2505_07239_amd as comet
    k = Case(3020, [(2, 20)], 4, 2, ldp=8)
    q, kv, table = k.dev["q"], k.dev["kv"], k.dev["table"]
    sizes = dict(n_tok=k.t, n_heads=4, n_kv_heads=2, page_size=16, max_q=2)
    for name in sizes:
        for far in (2 ** 32, -2 ** 32, 2 ** 31, 2 ** 32 + sizes[name]):
            with pytest.raises(ValueError):
                comet.KVBatch(q_start=q, kv_len=kv, block_table=table, **dict(sizes, **{name: far}))
    e, c, z = up(k.words(1, 8)), up(k.words(2, k.ld)), up(k.words(3, 8))
    f, x = up(k.f), up(k.x)
    rows, slots, cos = up(u64(3021, 1, 2, 8)), ints([0, 1]), up(u64(3021, 2, 5, 2))
    pools = up(u64(3021, 3, 4, 8)), up(u64(3021, 4, 4, 8))
    far = 2 ** 32
    calls = [lambda: ctx.attention_scores(far, k.batch, e, e, f, x, c), lambda: ctx.attention_scores(0, k.batch, e, e, f, x, c, far + 16),
             lambda: ctx.attention_values(far + 1, k.batch, c, c, f, x, z), lambda: ctx.attention_values(0, k.batch, c, c, f, x, z, far),
             lambda: ctx.attention_weights(far, k.batch, c, None, c, c, 5), lambda: ctx.attention_weights(0, k.batch, c, None, c, c, 5, far),
             lambda: ctx.cache_write(far, rows, rows, rows, slots, *pools), lambda: ctx.cache_read(far, *pools, slots),
             lambda: ctx.rotate_share(far, rows, slots, cos, cos, 2), lambda: ctx.rotate_share(0, rows, slots, cos, cos, 2, far),
             lambda: ctx.rotate_share(0, rows, slots, cos, cos, 2, 0, far)]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_weights_take_a_batch_without_a_page_table(ctx):
    """Of the batch the weights use lengths, heads and flags only."""
    say("weights without pages")
    k = Case(3030, [(2, 20), (1, 5)], 4, 2, mask=True)
    d_0, r, r2 = (up(k.words(i, k.ld)) for i in (1, 2, 3))
    outs = [(up(pattern(k.t, 4, k.ld)), up(pattern(k.t, 4))) for _ in (0, 1)]
    ctx.attention_weights(1, k.batch, d_0, None, r, r2, 7, 16, out=outs[0])
    bare = type(k.batch.struct)()
    ctypes.pointer(bare)[0] = k.batch.struct
    bare.block_table = None
    p = lambda t: t.data_ptr()
    assert ctx.lib.comet_attention_weights(ctx.h, 1, ctypes.byref(bare), k.ld, 16, 7, p(d_0), None, p(r), p(r2), None, p(outs[1][0]),
                                           p(outs[1][1])) == 0
    assert all(np.array_equal(down(a), down(b)) for a, b in zip(*outs))
    f, e = up(k.f), up(k.words(4, 8))
    assert ctx.lib.comet_attention_scores(ctx.h, 1, ctypes.byref(bare), 8, 8, len(k.f), k.ld, 16, p(e), p(e), p(f), p(f), p(d_0), None,
                                          p(outs[1][0]), None, 0) == -1


def test_results_over_operands_or_each_other_are_refused(ctx):
    """Where every order of reads and writes would be wrong."""
    say("results in one buffer")
    import paper_2505_07239_amd as comet
    k = Case(3040, [(2, 20)], 4, 2, ldp=32)
    assert k.ld == 32
    rows, pool, slots = up(u64(3041, 1, 2, 8)), up(u64(3041, 2, 4, 8)), ints([0, 1])
    c, e, a, f, x = up(k.words(1, 32)), up(k.words(2, 32)), up(k.words(3, 32)), up(k.f), up(k.x)
    calls = [lambda: ctx.cache_write(0, rows, rows, rows, slots, pool, pool),
             lambda: ctx.cache_read(0, pool, pool.clone(), slots, out=(rows, rows)),
             lambda: ctx.attention_weights(0, k.batch, c, None, c, c, 5, out=(c, c.view(-1)[:k.t * 4].view(k.t, 4)))]
    for call in (ctx.attention_scores, ctx.attention_values):
        calls += [lambda call=call, z=z: call(0, k.batch, e, a, f, x, c, 16, out=z) for z in (e, a)]
    for call in calls:
        with pytest.raises(comet.CometError) as err:
            call()
        assert err.value.code == -1


def test_a_prompt_bound_for_many_sequences(ctx):
    """The work of a batch follows its tokens: 16384 sequences of which any could be the one prompt of 1023 tokens of 128 heads
    over 8320 keys are 2^31 tiles of rows and keys when every sequence gets a prompt's."""
    say("prompt bound for many sequences")
    import paper_2505_07239_amd as comet
    n_seq, max_q, t, heads, page, d, ld = 16384, 1023, 1040, 128, 1664, 258, 8320
    lens = {3: (5, 40), 9000: (1, 70), 9001: (0, 9), 16383: (3, 2)}
    new, kv_len = np.zeros(n_seq, dtype=np.int32), np.zeros(n_seq, dtype=np.int32)
    for s, (n, kv) in lens.items():
        new[s], kv_len[s] = n, kv
    q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    table = (np.arange(n_seq, dtype=np.int32)[:, None] + np.arange(ld // page, dtype=np.int32)) % 3
    batch = comet.KVBatch(t, heads, 1, ints(q_start), ints(kv_len), ints(table), page, max_q)
    used, n = int(q_start[-1]), 80
    rows = list(oa.rows(q_start, kv_len, heads))
    f, x = (u64(3050, 1 + i, 3, page, 1, d) for i in (0, 1))
    e, a, c = u64(3050, 3, used, heads, d), u64(3050, 4, used, heads, d), u64(3050, 5, used, heads, n)
    filled = lambda v: torch.cat([up(v), torch.full((t - used,) + v.shape[1:], PATTERN, dtype=torch.int64, device="cuda")])
    z = torch.full((t, heads, ld), PATTERN, dtype=torch.int64, device="cuda")
    z[:used, :, :n] = up(c)
    ctx.attention_scores(1, batch, filled(e), filled(a), up(f), up(x), z, 16, out=z)
    assert np.array_equal(down(z[:used, :, :n].contiguous()), oa.scores(1, rows, e, a, f, x, table, c, 16, None, c))
    assert bool((z[:used, :, n:] == PATTERN).all()) and bool((z[used:] == PATTERN).all())


@pytest.mark.parametrize("heads,kvh", [(1, 1), (6, 2), (21, 1), (40, 1)])
@pytest.mark.parametrize("d", [40, 130, 320])
def test_where_the_tiles_of_prompts_lie(ctx, heads, kvh, d):
    """Prompts of every length between, behind and in front of single tokens and empty sequences, tokens before the first
    sequence and behind the last, more sequences than a wavefront has lanes."""
    say("tiles of prompts heads=%d kvh=%d d=%d" % (heads, kvh, d))
    few = max(16 * kvh // heads, 1)
    lens = [(0, 3), (few + 1, 40), (1, 9), (0, 0), (few + 1, few + 1), (few + 2, 7), (0, 5), (70, 90), (1, 33)]
    lens += [(s % 2, 2 + s) for s in range(75)] + [(few, 30), (33, 33)] + [(0, 1)] * 60 + [(few + 1, 20), (0, 4)]
    k = Case(3060 + d + heads, lens, heads, kvh, ldp=d, gap=5, pad=4, mask=d == 40)
    check_scores(ctx, k, d, 1, 16, True)
    check_values(ctx, k, d, 0, 16, True)
    k = Case(3070 + d + heads, [(0, 3)] * 70 + [(67, 67)], heads, kvh, ldp=d, max_q=30)
    check_scores(ctx, k, d, 0, 0, False)
    check_values(ctx, k, d, 1, 0, False)


def test_token_ranges_that_do_not_ascend(ctx):
    """What they give is unspecified; every access stays in the operands and the call ends."""
    say("ranges that do not ascend")
    k = Case(3080, [(20, 30), (1, 5)] + [(0, 2)] * 70 + [(25, 60)], 4, 2, ldp=64)
    e, a, c, z = (up(k.words(i, n)) for i, n in ((1, 64), (2, 64), (3, k.ld), (4, 64)))
    starts = list(k.q_start)
    for order in (starts[::-1], [k.t] * len(starts), [1 << 30] + starts[1:], [-5, 40, 3] + starts[3:]):
        k.dev["q"].copy_(ints(order))
        ctx.attention_scores(1, k.batch, e, a, up(k.f), up(k.x), c, 16)
        ctx.attention_values(1, k.batch, c, c, up(k.f), up(k.x), z, 16)
        ctx.attention_weights(1, k.batch, c, None, c, c, 5)
        torch.cuda.synchronize()
    k.dev["q"].copy_(ints(starts))
    check_scores(ctx, k, 64, 1, 16, True)
    check_values(ctx, k, 64, 1, 16, True)


DIGITS = [0x7F7F7F7F7F7F7F80, 0x7F7F7F7F7F7F7F7F]      # all eight signed digits -128, all 127


@pytest.mark.parametrize("d", [66, 128])
@pytest.mark.parametrize("kv", [8128, 8129, 16256])
@pytest.mark.parametrize("value", DIGITS)
def test_longest_pieces_of_keys(ctx, value, kv, d):
    """Digits of the largest magnitude in as many keys as one accumulator takes: 64 tokens of 256 heads, a tile of rows for every
    compute unit, so that cutting the keys further than the planes need does not pay.  Every row is c + 2 kv value^2."""
    say("longest pieces kv=%d d=%d %x" % (kv, d, value))
    import paper_2505_07239_amd as comet
    t, heads, page = 64, 256, 16
    ld = -(-kv // page) * page
    batch = comet.KVBatch(t, heads, heads, ints([0, t]), ints([kv]), torch.zeros((1, ld // page), dtype=torch.int32, device="cuda"), page, t,
                          causal=False)
    full = lambda *shape: torch.full(shape, value, dtype=torch.int64, device="cuda")
    w, pool, c = full(t, heads, ld), full(1, page, heads, d), up(u64(3090, 1, t, heads, d))
    got = ctx.attention_values(1, batch, w, w, pool, pool, c)
    assert torch.equal(got, c + up(np.array([2 * kv * value * value % 2 ** 64], dtype=np.uint64)))


@pytest.mark.parametrize("value", DIGITS)
@pytest.mark.parametrize("t,heads", [(1, 3), (3, 8), (2, 300)])
def test_longest_rows_of_keys(ctx, value, t, heads):
    """The same for scores: rows of 4096 words."""
    say("longest rows %d x %d" % (t, heads))
    import paper_2505_07239_amd as comet
    d, kv, ld = 4096, 130, 144
    batch = comet.KVBatch(t, heads, 1, ints([0, t]), ints([kv]), torch.zeros((1, 9), dtype=torch.int32, device="cuda"), 16, t, causal=False)
    full = lambda *shape: torch.full(shape, value, dtype=torch.int64, device="cuda")
    q, pool, c = full(t, heads, d), full(1, 16, 1, d), up(u64(3091, 1, t, heads, ld))
    got = ctx.attention_scores(1, batch, q, q, pool, pool, c)
    want = c + up(np.array([2 * d * value * value % 2 ** 64], dtype=np.uint64))
    want[:, :, kv:] = 0
    assert torch.equal(got, want)


@pytest.mark.parametrize("d,ldp", [(194, 194), (256, 256), (256, 260), (258, 258)])
@pytest.mark.parametrize("new,heads,kvh", [(1, 4, 1), (1, 16, 1), (5, 8, 1), (1, 40, 1), (20, 6, 1), (70, 2, 2)])
def test_widths_about_256(ctx, d, ldp, new, heads, kvh):
    """Where the rows' digits just fill the place they have, and just do not."""
    say("width %d of %d, %d tokens of %d heads" % (d, ldp, new, heads))
    k = Case(3100 + d + new + heads, [(new, new + 60), (new, 200)], heads, kvh, ldp=ldp)
    check_scores(ctx, k, d, 1, 16, True)
    check_values(ctx, k, d, 0, 16, True)


def test_pools_of_more_than_4_gb(ctx):
    """Slots beyond 2^32 bytes of a pool, written, read and multiplied with."""
    say("pools of more than 4 GB")
    import paper_2505_07239_amd as comet
    page, kvh, d, n_pages = 64, 8, 128, 9000                  # 64 * 8 KB a page: 4.7 GB
    assert n_pages * page * kvh * d * 8 > 2 ** 32 + 2 ** 28
    f, x = (torch.zeros((n_pages, page, kvh, d), dtype=torch.int64, device="cuda") for _ in (0, 1))
    last, first = n_pages - 1, 3
    kv, heads, new = 100, 16, 3
    slots = np.array([last * page + j for j in range(64)] + [first * page + j for j in range(36)], dtype=np.int32)
    d_0, d_1, b = (u64(3110, 1 + i, kv, kvh * d) for i in range(3))
    ctx.cache_write(1, up(d_0), up(d_1), up(b), up(slots), f, x)
    fv = d_0 + d_1
    e, a = ctx.cache_read(1, f, x, up(slots))
    assert np.array_equal(down(e), fv) and np.array_equal(down(a), b)
    assert int(f.ne(0).sum()) == kv * kvh * d                 # (no word of these is zero)
    small = [np.zeros((2, page, kvh, d), dtype=U) for _ in (0, 1)]
    for p, v in zip(small, (fv, b + fv)):
        p.reshape(2 * page, kvh * d)[:kv] = v
    rows, table = list(oa.rows([0, new], [kv], heads)), np.array([[0, 1]])
    batch = comet.KVBatch(new, heads, kvh, ints([0, new]), ints([kv]), ints([[last, first]]), page, new)
    e, a, c, z = u64(3111, 1, new, heads, d), u64(3111, 2, new, heads, d), u64(3111, 3, new, heads, 2 * page), u64(3111, 4, new, heads, d)
    got = ctx.attention_scores(0, batch, up(e), up(a), f, x, up(c), 16)
    assert np.array_equal(down(got), oa.scores(0, rows, e, a, *small, table, c, 16, None, np.zeros_like(c)))
    got = ctx.attention_values(0, batch, up(c), up(c), f, x, up(z), 16)
    assert np.array_equal(down(got), oa.values(0, rows, c, c, *small, table, z, 16, None, np.zeros_like(z)))


def test_graph_replayed_with_new_operands_in_place(ctx):
    """Queries, keys, values, pools, triple parts, pages, tokens of the sequences and active heads all change between replays."""
    say("graph with new operands")
    k = Case(3120, [(1, 40), (30, 70), (2, 9)], 4, 2, ldp=80, page=16, mask=True, pad=6, spare=1)
    d, n = 80, 6
    host = dict(e=k.words(1, d), a=k.words(2, d), c=k.words(3, k.ld), r=k.words(4, k.ld), r2=k.words(5, k.ld), m=k.words(6, k.ld),
                z=k.words(7, d), f=k.f, x=k.x)
    dev = {name: up(v) for name, v in host.items()}
    slots = ints(np.arange(n))

    def run():
        s = ctx.attention_scores(1, k.batch, dev["e"], dev["a"], dev["f"], dev["x"], dev["c"], 16, dev["r"])
        w, sums = ctx.attention_weights(1, k.batch, s, None, dev["r"], dev["r2"], 9, 16, dev["m"])
        o = ctx.attention_values(1, k.batch, w, dev["m"], dev["f"], dev["x"], dev["z"], 16)
        return [s, w, sums, o, *ctx.cache_read(1, dev["f"], dev["x"], slots, width=2 * d)]

    def want():
        rows = list(oa.rows(k.q_start, k.kv_len, 4, True, k.mask))
        none = lambda v: np.zeros_like(v)
        s = oa.scores(1, rows, host["e"], host["a"], host["f"], host["x"], k.table, host["c"], 16, host["r"], none(host["c"]))
        w, sums = oa.weights(1, rows, s, None, host["r"], host["r2"], 9, 16, host["m"], none(s), np.zeros((k.t, 4), dtype=U))
        o = oa.values(1, rows, w, host["m"], host["f"], host["x"], k.table, host["z"], 16, None, none(host["z"]))
        flat = lambda v: v.reshape(-1, 2 * d)
        at = down(slots.long()).astype(np.int64)
        none = np.zeros((n, 2 * d), dtype=U)
        return [s, w, sums, o, *oa.cache_read(1, flat(host["f"]), flat(host["x"]), at, none, none)]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        eager = run()
        assert all(np.array_equal(down(g), w) for g, w in zip(eager, want()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = run()
    for turn, lens in enumerate(([(1, 40), (30, 70), (2, 9)], [(0, 3), (1, 8), (30, 96)], [(16, 16), (15, 70), (8, 8)], [(1, 1), (1, 50), (1, 77)])):
        for i, name in enumerate(host):
            host[name] = u64(3121 + turn, i, *host[name].shape)
            dev[name].copy_(up(host[name]))
        k.q_start = [0] + list(np.cumsum([new for new, _ in lens]))
        k.kv_len = [kv for _, kv in lens]
        k.mask = (u64(3125 + turn, 1, k.t, 4) & U(1)).astype(np.uint8)
        k.table = k.table[::-1].copy()
        for name, v in (("q", k.q_start), ("kv", k.kv_len), ("table", k.table)):
            k.dev[name].copy_(ints(v))
        k.batch.tensors[3].copy_(up(k.mask))
        slots.copy_(ints(np.arange(n) * (turn + 2)))
        torch.cuda.synchronize()
        ctx.open(up(u64(3126, turn, 1000)), up(u64(3127, turn, 1000)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(down(h), w) for h, w in zip(held, want()))
