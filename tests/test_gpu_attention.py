"""Attention over a cache of shares on the GPU, word for word against the oracle: every output buffer starts
out with a pattern, so that what a call must leave alone shows too."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import attention as oa                    # noqa: E402
from workloads import rng                             # noqa: E402

U = np.uint64
PATTERN = 0x5A5A5A5A5A5A5A5A


def say(msg):
    print("[gpu-attention] " + msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_07239_amd as comet
    c = comet.Context(0)
    yield c
    c.close()


def up(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int64) if a.dtype == np.uint64 else a).cuda()


def down(t):
    torch.cuda.synchronize()
    return t.cpu().numpy().view(np.uint64)


def u64(seed, stream, *shape):
    return rng.uniform_u64(seed, stream, int(np.prod(shape))).reshape(shape)


def pattern(*shape):
    return np.full(shape, PATTERN, dtype=np.uint64)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32).cuda()


class Case:
    """A batch with its pools.  ``lens``: (new tokens, cached rows) per sequence."""

    def __init__(self, seed, lens, heads, kvh, page=16, ldp=8, causal=True, mask=False, pad=0, gap=0, max_q=None, spare=0):
        import paper_2505_07239_amd as comet
        self.seed, self.heads, self.kvh, self.page = seed, heads, kvh, page
        self.q_start = [gap]
        for new, _ in lens:
            self.q_start.append(self.q_start[-1] + new)
        self.kv_len = [kv for _, kv in lens]
        self.t = self.q_start[-1] + pad
        pages = max(max([-(-kv // page) for kv in self.kv_len] + [0]) + spare, 1)
        n = len(lens) * pages
        order = np.argsort(rng.uniform_u64(seed, 90, n + 2), kind="stable").astype(np.int32)
        self.table = order[:n].reshape(len(lens), pages)
        self.ld = pages * page
        self.f, self.x = (u64(seed, 91 + i, n + 2, page, kvh, ldp) for i in (0, 1))
        self.mask = (u64(seed, 93, self.t, heads) & U(1)).astype(np.uint8) if mask else None
        self.max_q = max(new for new, _ in lens) if max_q is None else max_q
        self.dev = dict(q=ints(self.q_start), kv=ints(self.kv_len), table=ints(self.table))
        self.batch = comet.KVBatch(self.t, heads, kvh, self.dev["q"], self.dev["kv"], self.dev["table"], page, self.max_q,
                                   causal=causal, head_mask=None if self.mask is None else up(self.mask))
        self.rows = list(oa.rows(self.q_start, self.kv_len, heads, causal, self.mask, self.max_q))

    def words(self, stream, *last):
        return u64(self.seed, stream, self.t, self.heads, *last)


def check_scores(ctx, k, d, party, bits, masked):
    e, a, c = k.words(1, d), k.words(2, d), k.words(3, k.ld)
    m = k.words(4, k.ld) if masked else None
    out = up(pattern(k.t, k.heads, k.ld))
    got = ctx.attention_scores(party, k.batch, up(e), up(a), up(k.f), up(k.x), up(c), bits, None if m is None else up(m), out=out)
    want = oa.scores(party, k.rows, e, a, k.f, k.x, k.table, c, bits, m, pattern(k.t, k.heads, k.ld))
    assert np.array_equal(down(got), want)


def check_values(ctx, k, d, party, bits, masked):
    e, a, c = k.words(5, k.ld), k.words(6, k.ld), k.words(7, d)
    m = k.words(8, d) if masked else None
    out = up(pattern(k.t, k.heads, d))
    got = ctx.attention_values(party, k.batch, up(e), up(a), up(k.f), up(k.x), up(c), bits, None if m is None else up(m), out=out)
    want = oa.values(party, k.rows, e, a, k.f, k.x, k.table, c, bits, m, pattern(k.t, k.heads, d))
    assert np.array_equal(down(got), want)


def check_weights(ctx, k, party, bits, masked, opened):
    d_0, d_1, r, r2 = (k.words(10 + i, k.ld) for i in range(4))
    m = k.words(14, k.ld) if masked else None
    d_1 = None if opened else d_1
    out = (up(pattern(k.t, k.heads, k.ld)), up(pattern(k.t, k.heads)))
    on = lambda v: None if v is None else up(v)
    got = ctx.attention_weights(party, k.batch, up(d_0), on(d_1), up(r), up(r2), -77, bits, on(m), out=out)
    want = oa.weights(party, k.rows, d_0, d_1, r, r2, 2 ** 64 - 77, bits, m, pattern(k.t, k.heads, k.ld), pattern(k.t, k.heads))
    assert np.array_equal(down(got[0]), want[0]) and np.array_equal(down(got[1]), want[1])


# one token and prompts, rows that see nothing, empty caches, padding, pages that end inside a tile
SHAPES = [
    dict(lens=[(1, 1)], heads=1, kvh=1),
    dict(lens=[(1, 0), (1, 17), (0, 5), (1, 33)], heads=4, kvh=2, pad=2),
    dict(lens=[(3, 2), (5, 5), (2, 40)], heads=6, kvh=2, gap=1, pad=3),
    dict(lens=[(20, 70)], heads=2, kvh=2, page=48, mask=True),
    dict(lens=[(70, 70), (33, 150)], heads=3, kvh=1, page=32),
    dict(lens=[(1, 700), (1, 81), (1, 300)], heads=8, kvh=1, page=64, spare=2),
    dict(lens=[(1, 1000)], heads=40, kvh=1, page=16, mask=True),
    dict(lens=[(17, 64), (64, 64)], heads=5, kvh=5, causal=False),
    dict(lens=[(9, 30)], heads=16, kvh=1, max_q=4),
    dict(lens=[(129, 129)], heads=1, kvh=1, page=16),
]


@pytest.mark.parametrize("n", range(len(SHAPES)))
@pytest.mark.parametrize("d,ldp", [(2, 2), (64, 64), (80, 96), (130, 130)])
def test_products(ctx, n, d, ldp):
    say("products %s d=%d ldp=%d" % (SHAPES[n], d, ldp))
    k = Case(2000 + 10 * n + d, ldp=ldp, **SHAPES[n])
    party = (n + d // 2) % 2
    check_scores(ctx, k, d, party, 16, n % 3 != 0)
    check_values(ctx, k, d, 1 - party, 13, n % 3 != 1)


@pytest.mark.parametrize("d,ldp,heads", [(576, 576, 16), (576, 576, 70), (512, 576, 16), (512, 576, 70), (322, 324, 3), (1000, 1002, 18), (4096, 4096, 2)])
def test_latent_rows(ctx, d, ldp, heads):
    """One row a token for all query heads; the values are the first words of the keys' rows."""
    say("latent d=%d ldp=%d heads=%d" % (d, ldp, heads))
    k = Case(2200 + d + heads, [(1, 130), (2, 77)], heads, 1, ldp=ldp)
    check_scores(ctx, k, d, 1, 0, False)
    check_values(ctx, k, d, 0, 16, True)


@pytest.mark.parametrize("heads,kvh,new", [(40, 1, 1), (20, 1, 1), (4, 2, 1), (2, 2, 24)])
@pytest.mark.parametrize("d,ldp", [(576, 576), (300, 320), (128, 128)])
def test_capacity_beyond_the_lengths(ctx, heads, kvh, new, d, ldp):
    """Calls are planned by what the operands could hold: rows of 4224 words of which a few are used, so that
    the variants for large batches run."""
    say("capacity heads=%d kvh=%d new=%d d=%d" % (heads, kvh, new, d))
    k = Case(2250 + d + heads, [(new, 50 + 13 * s) for s in range(8)], heads, kvh, page=64, ldp=ldp, spare=63)
    assert k.ld >= 4096
    check_scores(ctx, k, d, 1, 16, True)
    check_values(ctx, k, d, 0, 16, True)


@pytest.mark.parametrize("new,kv,heads,kvh,d", [(70, 1500, 2, 1, 64), (40, 1300, 2, 2, 80), (3, 2100, 8, 1, 128), (20, 9000, 1, 1, 16)])
def test_keys_in_pieces(ctx, new, kv, heads, kvh, d):
    """Few rows over long sequences: the keys are cut into pieces, some of which begin beyond what a row sees."""
    say("pieces new=%d kv=%d" % (new, kv))
    k = Case(2270 + d, [(new, kv), (new, new), (1, 700)], heads, kvh, page=32, ldp=d, mask=d == 64)
    check_scores(ctx, k, d, 0, 16, False)
    check_values(ctx, k, d, 1, 16, True)


def test_rows_far_apart(ctx):
    """Rows of a tile more than 2 GB apart: 40 tokens of one head, rows of 2^23 words."""
    say("far rows")
    import paper_2505_07239_amd as comet
    t, ld, d = 40, 1 << 23, 16
    q, kv, table = ints([0, t]), ints([50]), ints(np.zeros((1, ld // 16)))
    table[0, :4] = ints([2, 0, 1, 3])
    batch = comet.KVBatch(t, 1, 1, q, kv, table, 16, t)
    f, x = u64(2280, 1, 4, 16, 1, d), u64(2280, 2, 4, 16, 1, d)
    e, a = u64(2280, 3, t, 1, d), u64(2280, 4, t, 1, d)
    c, m = u64(2280, 5, t, 1, 64), u64(2280, 6, t, 1, 64)
    wide = [torch.zeros(t, 1, ld, dtype=torch.int64, device="cuda") for _ in range(3)]
    for w, v in zip(wide, (c, m, pattern(t, 1, 64))):
        w[:, :, :64] = up(v)
    out = ctx.attention_scores(1, batch, up(e), up(a), up(f), up(x), wide[0], 16, wide[1], out=wide[2])
    rows = list(oa.rows([0, t], [50], 1))
    want = oa.scores(1, rows, e, a, f, x, np.array([[2, 0, 1, 3]]), c, 16, m, pattern(t, 1, 64))
    assert np.array_equal(down(out[:, :, :64].contiguous()), want)
    assert not bool(out[:, :, 64:].any())
    z = u64(2280, 7, t, 1, d)
    got = ctx.attention_values(0, batch, out, wide[1], up(f), up(x), up(z), 16)
    assert np.array_equal(down(got), oa.values(0, rows, want, m, f, x, np.array([[2, 0, 1, 3]]), z, 16, None, np.zeros_like(z)))


def test_more_workgroups_than_one_launch_takes(ctx):
    """A bound on a sequence's tokens that one prompt could fill, for many sequences: more than 2^32 threads."""
    say("many workgroups")
    import paper_2505_07239_amd as comet
    n_seq, t, heads, page, d, new = 1100, 1030, 128, 1024, 320, 9
    q_start, kv_len = np.zeros(n_seq + 1, dtype=np.int32), np.zeros(n_seq, dtype=np.int32)
    q_start[1:], q_start[601:], q_start[1100:] = 3, 8, 9
    kv_len[0], kv_len[600], kv_len[1099] = 40, 5, 150
    table = np.arange(n_seq, dtype=np.int32).reshape(n_seq, 1) % 3
    table[600], table[1099] = 2, 1
    batch = comet.KVBatch(t, heads, 1, ints(q_start), ints(kv_len), ints(table), page, t)
    rows = list(oa.rows(q_start, kv_len, heads))
    f, x = u64(2300, 1, 3, page, 1, 512), u64(2300, 2, 3, page, 1, 512)

    def wide(stream, last):
        """[t, heads, last] words, random for the tokens of the batch, the pattern behind them."""
        small = pattern(new, heads, last) if stream is None else u64(2300, stream, new, heads, last)
        all_of = torch.full((t, heads, last), PATTERN, dtype=torch.int64, device="cuda")
        all_of[:new] = up(small)
        return small, all_of

    def same(got, want):
        assert np.array_equal(down(got[:new].contiguous()), want)
        assert bool((got[new:] == PATTERN).all())

    (e, e_), (a, a_), (c, c_), (z, z_) = wide(3, d), wide(4, d), wide(5, page), wide(None, page)
    same(ctx.attention_scores(1, batch, e_, a_, up(f), up(x), c_, 16, out=z_), oa.scores(1, rows, e, a, f, x, table, c, 16, None, z))
    (w, w_), (v, v_), (c, c_), (z, z_) = wide(6, page), wide(7, page), wide(8, 512), wide(None, 512)
    same(ctx.attention_values(0, batch, w_, v_, up(f), up(x), c_, 16, out=z_), oa.values(0, rows, w, v, f, x, table, c, 16, None, z))
    (z, z_), (sums, sums_) = wide(None, page), wide(None, 1)
    got = ctx.attention_weights(1, batch, w_, None, v_, w_, 5, 16, out=(z_, sums_[:, :, 0].contiguous()))
    want = oa.weights(1, rows, w, None, v, w, 5, 16, None, z, sums[:, :, 0])
    same(got[0], want[0]), same(got[1], want[1])


def test_more_rows_of_weights_than_one_launch_takes(ctx):
    say("many rows")
    import paper_2505_07239_amd as comet
    t, heads = (1 << 19) + 5, 128
    batch = comet.KVBatch(t, heads, 1, ints([0, t]), ints([2]), ints([[0]]), 16, t, causal=False)
    gen = torch.Generator(device="cuda").manual_seed(2310)
    u, r, r2 = (torch.randint(-2 ** 63, 2 ** 63 - 1, (t, heads, 2), dtype=torch.int64, device="cuda", generator=gen) for _ in range(3))
    out, sums = ctx.attention_weights(0, batch, u, None, r, r2, 3, 7)
    want = (r2 + 2 * (u + 3) * r) >> 7
    assert torch.equal(out, want) and torch.equal(sums, want[:, :, 0] + want[:, :, 1])


@pytest.mark.parametrize("lens,max_q", [([(9, 30), (1, 3), (0, 4), (2, 8)], 4), ([(1, 900), (0, 0), (0, 7), (40, 700), (1, 1), (0, 9)], None),
                                        ([(0, 3), (30, 30)] + [(1, 20 * s) for s in range(20)], None)])
@pytest.mark.parametrize("heads,kvh,d", [(4, 2, 80), (40, 1, 80), (20, 1, 320), (3, 3, 40)])
def test_prompts_among_single_tokens(ctx, lens, max_q, heads, kvh, d):
    say("mixed %s heads=%d d=%d" % (lens, heads, d))
    k = Case(2320 + len(lens) + heads, lens, heads, kvh, ldp=d, gap=2, pad=3, max_q=max_q, spare=20)
    check_weights(ctx, k, 1, 16, True, False)
    check_scores(ctx, k, d, 0, 16, True)
    check_values(ctx, k, d, 1, 16, True)


@pytest.mark.parametrize("d", [64, 102])
def test_many_short_prompts(ctx, d):
    """Row tiles of 64 for every compute unit over short keys."""
    say("short prompts d=%d" % d)
    k = Case(2340 + d, [(17 + s % 3, 18 + s % 7) for s in range(96)], 6, 3, ldp=d, pad=1, mask=d == 102)
    check_scores(ctx, k, d, 1, 16, True)
    check_values(ctx, k, d, 0, 16, False)


@pytest.mark.parametrize("new", [1, 30])
def test_no_pages(ctx, new):
    """A cache without pages: no row sees anything, the values are what their masks say."""
    say("no pages")
    import paper_2505_07239_amd as comet
    t, heads, d, ld = 2 * new, 2, 6, 16
    batch = comet.KVBatch(t, heads, 1, ints([0, new, t]), ints([3, 0]), torch.zeros((2, 0), dtype=torch.int32, device="cuda"), 16, new)
    pool = torch.zeros((0, 16, 1, 8), dtype=torch.int64, device="cuda")
    e, c, m, z = u64(2330, 1, t, heads, ld), u64(2330, 2, t, heads, d), u64(2330, 3, t, heads, d), pattern(t, heads, ld)
    got = ctx.attention_values(1, batch, up(e), up(e), pool, pool, up(c), 16, up(m))
    assert np.array_equal(down(got), oa.rescale(1, c, 16) - m)
    assert np.array_equal(down(ctx.attention_scores(1, batch, up(c), up(c), pool, pool, up(e), 16, out=up(z))), z)
    w, sums = ctx.attention_weights(0, batch, up(e), None, up(e), up(e), 1, out=(up(z), up(pattern(t, heads))))
    assert np.array_equal(down(w), z) and not down(sums).any()


def test_two_contexts_on_two_streams(ctx):
    """Calls of two contexts in flight together share nothing."""
    import paper_2505_07239_amd as comet
    cases = [Case(2290 + i, [(1, 3000 - 500 * i), (1, 900)], 8, 2, page=64, ldp=64) for i in (0, 1)]
    both, streams = [ctx, comet.Context(0)], [torch.cuda.Stream(), torch.cuda.Stream()]
    ops = [[up(k.words(5, k.ld)), up(k.words(6, k.ld)), up(k.f), up(k.x), up(k.words(7, 64))] for k in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(both[i].attention_values(i, cases[i].batch, *ops[i], 16))
    torch.cuda.synchronize()
    for i, k in enumerate(cases):
        want = oa.values(i, k.rows, k.words(5, k.ld), k.words(6, k.ld), k.f, k.x, k.table, k.words(7, 64), 16, None,
                         np.zeros((k.t, k.heads, 64), dtype=U))
        assert all(np.array_equal(down(o), want) for o in outs[i])
    both[1].close()


@pytest.mark.parametrize("value", [0, 2 ** 64 - 1, 1 << 63, 0x7F7F7F7F7F7F7F7F, 0x8080808080808080])
def test_words_at_the_ends_of_the_ring(ctx, value):
    """Digits of the largest magnitude over a long contraction: partial sums must not overflow."""
    say("ends %x" % value)
    k = Case(2300, [(1, 9000), (2, 5)], 2, 1, page=512, ldp=64)
    k.f[:], k.x[:] = U(value), U(value)
    seen, k.words = k.words, lambda stream, *last: np.full((k.t, k.heads) + last, value, dtype=np.uint64)
    check_values(ctx, k, 64, 1, 0, False)
    check_scores(ctx, k, 64, 0, 62, True)
    k.words = seen


@pytest.mark.parametrize("n", range(len(SHAPES)))
@pytest.mark.parametrize("party", [0, 1])
def test_weights(ctx, n, party):
    say("weights %s party=%d" % (SHAPES[n], party))
    k = Case(2400 + n, **SHAPES[n])
    check_weights(ctx, k, party, (0, 16, 62)[n % 3], n % 2 == 0, n % 4 == 1)


def test_in_place_results(ctx):
    """Z over C, Z over M, weights over any of their inputs."""
    k = Case(2500, [(20, 70), (1, 130)], 4, 2, ldp=64)
    d = 64
    e, a, c, m = k.words(1, d), k.words(2, d), k.words(3, k.ld), k.words(4, k.ld)
    for over in ("c", "m"):
        cd, md = up(c), up(m)
        out = cd if over == "c" else md
        ctx.attention_scores(1, k.batch, up(e), up(a), up(k.f), up(k.x), cd, 16, md, out=out)
        assert np.array_equal(down(out), oa.scores(1, k.rows, e, a, k.f, k.x, k.table, c, 16, m, c if over == "c" else m))
    e, a, c, m = k.words(1, k.ld), k.words(2, k.ld), k.words(3, d), k.words(4, d)
    for over in ("c", "m"):
        cd, md = up(c), up(m)
        out = cd if over == "c" else md
        ctx.attention_values(0, k.batch, up(e), up(a), up(k.f), up(k.x), cd, 16, md, out=out)
        assert np.array_equal(down(out), oa.values(0, k.rows, e, a, k.f, k.x, k.table, c, 16, m, c if over == "c" else m))
    ops = [k.words(10 + i, k.ld) for i in range(5)]
    for over in range(5):
        dev = [up(v) for v in ops]
        sums = torch.zeros(k.t, k.heads, dtype=torch.int64, device="cuda")
        ctx.attention_weights(1, k.batch, dev[0], dev[1], dev[2], dev[3], 5, 16, dev[4], out=(dev[over], sums))
        want = oa.weights(1, k.rows, ops[0], ops[1], ops[2], ops[3], 5, 16, ops[4], ops[over], np.zeros((k.t, k.heads), dtype=U))
        assert np.array_equal(down(dev[over]), want[0]) and np.array_equal(down(sums), want[1])


def test_what_does_not_fit_stays_in_bounds(ctx):
    """Page ids outside the pools read page 0, lengths beyond the operands end there, tokens outside every sequence
    are left alone."""
    k = Case(2600, [(2, 40), (3, 30)], 2, 1, ldp=64)
    k.dev["table"][0, 1] = 1 << 20
    k.dev["table"][1, 0] = -1
    k.table = k.table.copy()
    k.table[0, 1] = k.table[1, 0] = 0
    check_scores(ctx, k, 64, 0, 16, True)
    check_values(ctx, k, 64, 1, 16, True)
    k.dev["kv"][0], k.dev["kv"][1] = 1 << 30, -5
    k.rows = list(oa.rows(k.q_start, [k.ld, 0], k.heads))
    check_scores(ctx, k, 64, 1, 16, False)
    check_values(ctx, k, 64, 0, 16, False)
    check_weights(ctx, k, 1, 16, True, False)
    k.dev["q"][2] = 1000                                     # ends beyond the tokens there are
    k.dev["q"][0] = -3
    k.rows = list(oa.rows([0, k.q_start[1], k.t], [k.ld, 0], k.heads, max_q=k.max_q))
    check_scores(ctx, k, 64, 1, 16, False)
    check_values(ctx, k, 64, 0, 16, False)


@pytest.mark.parametrize("t,width", [(1, 1), (3, 7), (5, 64), (40, 2050), (300, 576)])
@pytest.mark.parametrize("party", [0, 1])
def test_cache_rows(ctx, t, width, party):
    say("cache rows %d x %d" % (t, width))
    seed, n = 2700 + t + width, 2 * t + 1
    slots = np.argsort(rng.uniform_u64(seed, 1, n), kind="stable").astype(np.int32)[:t]
    if t > 2:
        slots[1], slots[2] = -1, n
    d0, d1, b = (u64(seed, 2 + i, t, width) for i in range(3))
    f, x = u64(seed, 5, n, width), u64(seed, 6, n, width)
    fd, xd = up(f), up(x)
    ctx.cache_write(party, up(d0), up(d1), up(b), up(slots), fd, xd)
    f, x = oa.cache_write(party, d0, d1, b, slots, f, x)
    assert np.array_equal(down(fd), f) and np.array_equal(down(xd), x)
    again = np.concatenate([slots, slots[:1], slots[:1]])     # a slot may be read any number of times
    out = tuple(up(pattern(t + 2, width)) for _ in (0, 1))
    e, a = ctx.cache_read(party, fd, xd, up(again), out=out)
    want = oa.cache_read(party, f, x, again, pattern(t + 2, width), pattern(t + 2, width))
    assert np.array_equal(down(e), want[0]) and np.array_equal(down(a), want[1])


def test_no_tokens(ctx):
    none = torch.zeros((0, 8), dtype=torch.int64, device="cuda")
    pool = up(u64(2750, 1, 4, 8))
    slots = ints(np.zeros(0, dtype=np.int32))
    ctx.cache_write(0, none, none, none, slots, pool, pool.clone())
    assert ctx.cache_read(1, pool, pool, slots)[0].shape == (0, 8)
    table = up(u64(2750, 2, 3, 2))
    assert ctx.rotate_share(0, none, slots, table, table, 2).shape == (0, 8)


@pytest.mark.parametrize("t,heads,d,rot", [(1, 1, 2, 2), (1, 32, 128, 128), (5, 3, 10, 6), (7, 2, 9, 4), (33, 4, 80, 80), (2, 3, 6, 0),
                                           (6, 1, 576, 64), (300, 5, 64, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate(ctx, t, heads, d, rot, interleaved):
    say("rotate %s" % ((t, heads, d, rot, interleaved),))
    seed = 2800 + t + d + rot
    wide, off = u64(seed, 1, t, heads * d + 5), (0, 3, 2)[(t + d) % 3]
    cos, sin = u64(seed, 2, 50, rot // 2), u64(seed, 3, 50, rot // 2)
    pos = (u64(seed, 4, t) % U(50)).astype(np.int32)
    if t > 2:
        pos[1], pos[2] = 50, -1                              # outside the table: read as 0
    m = u64(seed, 5, t, heads * d)
    x = up(wide)[:, off:off + heads * d]
    for party, shift, bits, masked in ((0, 16, 16, True), (1, 16, 16, False), (1, 0, 62, True), (0, 62, 0, False)):
        got = ctx.rotate_share(party, x, up(pos), up(cos), up(sin), heads, shift, bits, up(m) if masked else None, interleaved)
        want = oa.rotate(party, wide[:, off:off + heads * d], pos, cos, sin, heads, shift, bits, m if masked else None, interleaved)
        assert np.array_equal(down(got), want)
    md = up(m)                                               # the result over its mask
    ctx.rotate_share(1, x, up(pos), up(cos), up(sin), heads, 16, 16, md, interleaved, out=md)
    assert np.array_equal(down(md), oa.rotate(1, wide[:, off:off + heads * d], pos, cos, sin, heads, 16, 16, m, interleaved))


# ---------------------------------------------------------------------------
# one layer's attention, both parties
# ---------------------------------------------------------------------------

class Layer:
    """Attention of both parties from projected queries, keys and values (scale 2^32) to unnormalised outputs
    and row sums, every opening an addition of what the parties send each other."""

    def __init__(self, seed, lens, heads, kvh, d, page=16):
        self.k = Case(seed, lens, heads, kvh, page=page, ldp=d)
        k = self.k
        self.d, t = d, k.t
        gauss = lambda stream, *shape: rng.gaussian_f64(seed, stream, int(np.prod(shape))).reshape(shape)
        self.plain = [gauss(1 + i, t, n * d) for i, n in enumerate((heads, kvh, kvh))]
        split = lambda stream, v: (lambda r: [r, v - r])(u64(seed, stream, *v.shape))
        fixed = lambda v, s: np.round(v * 2.0 ** s).astype(np.int64).view(np.uint64)
        self.x = [split(10 + i, fixed(p, 32)) for i, p in enumerate(self.plain)]
        angle = np.arange(256)[:, None] * 10000.0 ** (-2.0 * np.arange(d // 2) / d)
        self.cos, self.sin = fixed(np.cos(angle), 16), fixed(np.sin(angle), 16)
        self.angle = angle
        # a token's place in its sequence, and the slots of the new rows
        self.pos, self.slots = np.zeros(t, dtype=np.int32), np.full(t, -1, dtype=np.int32)
        for s, (new, kv) in enumerate(lens):
            for j in range(new):
                p = kv - new + j
                self.pos[k.q_start[s] + j] = p
                self.slots[k.q_start[s] + j] = k.table[s, p // page] * page + p % page
        # what is cached already: plain values in fixed point, masked
        n = k.f.shape[0]
        self.pool = [fixed(gauss(20 + i, n, page, kvh, d), 16) for i in (0, 1)]
        self.pool_b = [[u64(seed, 30 + 2 * i + p, n, page, kvh, d) for p in (0, 1)] for i in (0, 1)]
        self.new_b = [[u64(seed, 40 + 2 * i + p, t, kvh * d) for p in (0, 1)] for i in (0, 1)]
        self.a_q = [u64(seed, 50 + p, t, heads, d) for p in (0, 1)]
        self.r = [u64(seed, 52 + p, t, heads, k.ld) for p in (0, 1)]
        self.r2 = split(54, (self.r[0] + self.r[1]) * (self.r[0] + self.r[1]))
        self.a_w = [u64(seed, 55 + p, t, heads, k.ld) for p in (0, 1)]
        b = [self.pool_b[i][0] + self.pool_b[i][1] for i in (0, 1)]
        for i in (0, 1):
            for j, slot in enumerate(self.slots):
                if slot >= 0:
                    b[i][slot // page, slot % page] = (self.new_b[i][0] + self.new_b[i][1])[j].reshape(kvh, d)
        self.c_s = split(60, np.zeros((t, heads, k.ld), dtype=U))
        self.c_o = split(61, np.zeros((t, heads, d), dtype=U))
        a_q, a_w = self.a_q[0] + self.a_q[1], self.a_w[0] + self.a_w[1]
        group = heads // kvh
        for s, j, h, v in k.rows:                            # C = A B on what the rows see
            self.c_s[1][j, h, :v] += oa.cached(b[0], k.table, s, v, h // group, d) @ a_q[j, h]
            self.c_o[1][j, h] += a_w[j, h, :v] @ oa.cached(b[1], k.table, s, v, h // group, d)
        self.bias = 5 << 16
        self.none = np.zeros((256, 0), dtype=U)              # the table of values: rescaled and masked only
        self.f = [self.pool[i] - self.pool_b[i][0] - self.pool_b[i][1] for i in (0, 1)]
        self.xs = [[self.pool_b[i][0], self.pool_b[i][1] + self.f[i]] for i in (0, 1)]

    def run(self, make, ops):
        """``make``: array to operand; ``ops``: the calls (GPU or oracle).  [(outputs, sums)] of the two parties."""
        k, both, t = self.k, (0, 1), self.k.t
        page, kvh, d = k.page, k.kvh, self.d
        heads = k.heads
        pools = []
        for i in both:                                       # keys and values into the cache
            cos, sin = (self.cos, self.sin) if i == 0 else (self.none, self.none)
            send = [ops.rotate(p, make(self.x[1 + i][p]), self.pos, cos, sin, kvh, 16, 16, make(self.new_b[i][p])) for p in both]
            pools.append([ops.write(p, send, make(self.new_b[i][p]), self.slots, make(self.f[i]), make(self.xs[i][p])) for p in both])
        send = [ops.rotate(p, make(self.x[0][p]), self.pos, self.cos, self.sin, heads, 16, 16,
                           make(self.a_q[p]).reshape(t, -1)) for p in both]
        e = ops.open(send).reshape(t, heads, d)
        send = [ops.scores(p, k, e, make(self.a_q[p]), *pools[0][p], make(self.c_s[p]), 16, make(self.r[p])) for p in both]
        made = [ops.weights(p, k, send, make(self.r[p]), make(self.r2[p]), self.bias, 16, make(self.a_w[p])) for p in both]
        e = ops.open([m[0] for m in made])
        return [(ops.values(p, k, e, make(self.a_w[p]), *pools[1][p], make(self.c_o[p]), 16), made[p][1]) for p in both]


class OracleOps:
    def rotate(self, p, x, pos, cos, sin, heads, shift, bits, m):
        return oa.rotate(p, x, pos, cos, sin, heads, shift, bits, m)

    def open(self, send):
        return send[0] + send[1]

    def write(self, p, send, b, slots, f, x):
        shape = f.shape
        flat = lambda v: v.reshape(shape[0] * shape[1], -1)
        return [v.reshape(shape) for v in oa.cache_write(p, send[0], send[1], b, slots, flat(f), flat(x))]

    def scores(self, p, k, e, a, f, x, c, bits, m):
        return oa.scores(p, k.rows, e, a, f, x, k.table, c, bits, m, np.zeros_like(c))

    def weights(self, p, k, send, r, r2, bias, bits, m):
        return oa.weights(p, k.rows, send[0], send[1], r, r2, bias, bits, m, np.zeros_like(r), np.zeros(r.shape[:2], dtype=U))

    def values(self, p, k, e, a, f, x, c, bits):
        return oa.values(p, k.rows, e, a, f, x, k.table, c, bits, None, np.zeros_like(c))


class GpuOps:
    """Operands that a caller keeps are made once per array, so that a captured run finds them where they were."""

    def __init__(self, ctx):
        self.ctx, self.kept = ctx, {}

    def make(self, a):
        key = (a.ctypes.data, a.shape)
        if key not in self.kept:
            self.kept[key] = (up(a), a)
        return self.kept[key][0]

    def rotate(self, p, x, pos, cos, sin, heads, shift, bits, m):
        return self.ctx.rotate_share(p, x, self.make(pos), self.make(cos), self.make(sin), heads, shift, bits, m)

    def open(self, send):
        return self.ctx.open(send[0], send[1])

    def write(self, p, send, b, slots, f, x):
        f, x = f.clone(), x.clone()
        self.ctx.cache_write(p, send[0], send[1], b, self.make(slots), f, x)
        return [f, x]

    def scores(self, p, k, e, a, f, x, c, bits, m):
        return self.ctx.attention_scores(p, k.batch, e, a, f, x, c, bits, m)

    def weights(self, p, k, send, r, r2, bias, bits, m):
        return self.ctx.attention_weights(p, k.batch, send[0], send[1], r, r2, bias, bits, m)

    def values(self, p, k, e, a, f, x, c, bits):
        return self.ctx.attention_values(p, k.batch, e, a, f, x, c, bits)


@pytest.mark.parametrize("lens,heads,kvh,d", [([(1, 50), (1, 7)], 4, 2, 16), ([(12, 12), (5, 40)], 2, 2, 8)])
def test_layer_of_both_parties(ctx, lens, heads, kvh, d):
    """The oracle's run against plain attention in float64, the GPU's against the oracle's, word for word.

    With u = 2^-16: a rescaling is off by less than u, so a cached or rotated word by at most
    r = u (3 + (|x_p| + |x_q|) / 2) (see the rotation's own test), a score by d r (|q| + |k| + r) + u, a weight by
    (2 |s + c| + its error) times that + u, an output by the sums over a row of these, and u."""
    y = Layer(2900 + d, lens, heads, kvh, d)
    want = y.run(lambda a: a, OracleOps())
    ops = GpuOps(ctx)
    got = y.run(ops.make, ops)
    for p in (0, 1):
        assert np.array_equal(down(got[p][0]), want[p][0]) and np.array_equal(down(got[p][1]), want[p][1])
    k, u = y.k, 2.0 ** -16
    real = lambda v: v.view(np.int64) / 65536.0
    turned = []
    for i, n in ((0, heads), (1, kvh)):
        x = y.plain[i].reshape(k.t, n, d)
        c, s = np.cos(y.angle[y.pos])[:, None], np.sin(y.angle[y.pos])[:, None]
        turned.append(np.concatenate([x[..., :d // 2] * c - x[..., d // 2:] * s, x[..., d // 2:] * c + x[..., :d // 2] * s], -1))
    pools = [real(p).copy() for p in y.pool]
    new = [turned[1], y.plain[2].reshape(k.t, kvh, d)]
    for i in (0, 1):
        for j, slot in enumerate(y.slots):
            if slot >= 0:
                pools[i][slot // k.page, slot % k.page] = new[i][j]
    top = max(np.abs(v).max() for v in y.plain)
    r = u * (3 + top)
    out, sums = real(want[0][0] + want[1][0]), real(want[0][1] + want[1][1])
    flat = lambda i, s, v, h: pools[i][k.table[s]].reshape(-1, kvh, d)[:v, h // (heads // kvh)]
    for s, j, h, v in k.rows:
        keys, vals = flat(0, s, v, h), flat(1, s, v, h)
        q = turned[0][j, h]
        score = keys @ q
        ds = r * (np.abs(keys).sum(1) + np.abs(q).sum() + d * r) + u
        w = (score + 5.0) ** 2
        dw = (2 * np.abs(score + 5.0) + ds) * ds + u
        do = (dw[:, None] * (np.abs(vals) + r) + w[:, None] * r).sum(0) + u
        assert (np.abs(out[j, h] - w @ vals) <= do).all()
        assert abs(sums[j, h] - w.sum()) <= dw.sum()


def test_layer_replayed_from_a_graph_on_another_stream(ctx):
    """Captured once and replayed with new queries, keys and lengths in place, eager work in between."""
    y = Layer(2950, [(1, 40), (1, 21), (2, 9)], 4, 2, 16)
    ops = GpuOps(ctx)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        eager = y.run(ops.make, ops)
        want = [[down(v) for v in both] for both in eager]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = y.run(ops.make, ops)
    full = list(y.k.kv_len)
    for turn, lens in enumerate((full, full, [40, 20, 0], full)):
        y.k.dev["kv"].copy_(ints(lens))
        torch.cuda.synchronize()
        ops.open([up(u64(2951, turn, 1000)), up(u64(2952, turn, 1000))])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if lens == full:
            assert all(np.array_equal(down(held[p][i]), want[p][i]) for p in (0, 1) for i in (0, 1))
        else:
            fresh = y.run(ops.make, ops)
            assert all(np.array_equal(down(held[p][i]), down(fresh[p][i])) for p in (0, 1) for i in (0, 1))


def test_latent_rows_expanded_by_a_share_product(ctx):
    """The expanded form: latent rows read back are E and A_i of the product with the expanding weights."""
    import oracle as co
    t, width, n = 20, 64, 96
    f, x = u64(2960, 1, 40, width), [u64(2960, 2 + i, 40, width) for i in (0, 1)]
    slots = np.arange(39, 39 - t, -1).astype(np.int32)
    fw, bw, c = u64(2960, 4, width, n), [u64(2960, 5 + i, width, n) for i in (0, 1)], [u64(2960, 7 + i, t, n) for i in (0, 1)]
    idx = ints(np.arange(n // 8))
    for p in (0, 1):
        e, a = ctx.cache_read(p, up(f), up(x[p]), up(slots))
        z = ctx.somm_share(p, 8, idx, None, n // 8, e, up(fw), a, up(bw[p]), up(c[p]))
        want = co.beaver_share(p, f[slots], fw, x[p][slots] - f[slots] * U(p), bw[p], c[p])
        assert np.array_equal(down(z), want)


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------

def test_refusals(ctx):
    import paper_2505_07239_amd as comet
    k = Case(2990, [(2, 20)], 4, 2, ldp=8)
    e, a, c = (up(k.words(1 + i, n)) for i, n in enumerate((8, 8, k.ld)))
    f, x = up(k.f), up(k.x)
    good = lambda **o: dict(dict(party=0, batch=k.batch, e=e, a_i=a, f_pool=f, x_pool=x, c_i=c, frac_bits=16), **o)
    ctx.attention_scores(**good())
    for bad in (dict(e=e.float()), dict(e=e.cpu()), dict(a_i=a.transpose(0, 1)), dict(f_pool=f.to(torch.int32))):
        with pytest.raises(TypeError):
            ctx.attention_scores(**good(**bad))
    for bad in (dict(e=e[:, :, :6].contiguous()), dict(f_pool=f[:, :8].contiguous()), dict(c_i=c[:1].contiguous()),
                dict(x_pool=x[:1].contiguous()), dict(m_i=e), dict(out=e)):
        with pytest.raises(ValueError):
            ctx.attention_scores(**good(**bad))
    odd = up(k.words(9, k.ld + 1))
    for bad in (dict(party=2), dict(frac_bits=63), dict(frac_bits=-1), dict(c_i=odd),
                dict(e=up(k.words(1, 7)), a_i=up(k.words(1, 7))), dict(e=up(k.words(1, 10)), a_i=up(k.words(1, 10)))):
        with pytest.raises(comet.CometError) as err:
            ctx.attention_scores(**good(**bad))
        assert err.value.code == -1
    with pytest.raises(comet.CometError) as err:             # no room for a key
        ctx.attention_weights(0, k.batch, *[torch.zeros((k.t, 4, 0), dtype=torch.int64, device="cuda")] * 4, 0)
    assert err.value.code == -1
    need = comet.workspace_bytes(comet.OP_VALUES, 8, 20000, 64, 0)
    assert need >= 3 * 8 * 64 * 8 and comet.workspace_bytes(comet.OP_SCORES, 8, 64, 20000, 0) == 0
    wide = up(k.words(1, 4098))
    big = torch.zeros((1, 16, 2, 4098), dtype=torch.int64, device="cuda")
    with pytest.raises(comet.CometError) as err:
        ctx.attention_scores(**good(e=wide, a_i=wide, f_pool=big, x_pool=big))
    assert err.value.code == -3
    q, kv, table = k.dev["q"], k.dev["kv"], k.dev["table"]
    for args in ((k.t, 4, 3, q, kv, table, 16, 2), (k.t, 4, 0, q, kv, table, 16, 2)):
        with pytest.raises(comet.CometError) as err:
            ctx.attention_weights(0, comet.KVBatch(*args), c, c, c, c, 0)
        assert err.value.code == -1
    with pytest.raises(comet.CometError):
        ctx.attention_weights(0, comet.KVBatch(k.t, 4, 2, q, kv, table, 24, 2), c, c, c, c, 0)
    with pytest.raises(ValueError):
        comet.KVBatch(k.t, 4, 2, q[:1], kv, table, 16, 2)
    with pytest.raises(TypeError):
        comet.KVBatch(k.t, 4, 2, q.long(), kv, table, 16, 2)
    with pytest.raises(ValueError):
        comet.KVBatch(k.t, 4, 2, q, kv, table, 16, 2, head_mask=torch.ones(1, 4, dtype=torch.uint8, device="cuda"))
    rows, slots = up(u64(2991, 1, 2, 8)), ints([0, 1])
    pool = up(u64(2991, 2, 4, 8))
    for bad in ((rows, rows[:1].contiguous(), rows, slots, pool, pool), (rows, rows, rows, slots[:1], pool, pool),
                (rows, rows, rows, slots, pool, pool[:3].contiguous())):
        with pytest.raises(ValueError):
            ctx.cache_write(0, *bad)
    with pytest.raises(comet.CometError):
        ctx.cache_write(2, rows, rows, rows, slots, pool, pool.clone())
    with pytest.raises(ValueError):
        ctx.cache_read(0, pool, pool, slots, width=4, out=(rows, rows.clone()))
    cos = up(u64(2991, 3, 5, 2))
    with pytest.raises(ValueError):
        ctx.rotate_share(0, rows, slots, cos, cos, 3)
    with pytest.raises(ValueError):
        ctx.rotate_share(0, rows, slots[:1], cos, cos, 2)
    with pytest.raises(comet.CometError):
        ctx.rotate_share(0, rows, slots, up(u64(2991, 4, 5, 3)), up(u64(2991, 5, 5, 3)), 2)
    with pytest.raises(comet.CometError):
        ctx.rotate_share(0, rows, slots, cos, cos, 2, out=rows)
    with pytest.raises(comet.CometError):
        ctx.rotate_share(0, rows, slots, cos[:0], cos[:0], 2)
