"""The oracle of attention over a cache of shares, pinned by what its formulas must give: reconstructed
products, squared weights and rotations against the plain computation, and the refusals that need no GPU."""
import ctypes
import os
import re

import numpy as np
import pytest

import oracle as co
from oracle import attention as oa
from workloads import rng

U = np.uint64
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def u64(seed, stream, *shape):
    return rng.uniform_u64(seed, stream, int(np.prod(shape))).reshape(shape)


def signed(x):
    return x.view(np.int64)


def test_rescale_matches_the_shares_own_rule():
    z = u64(900, 1, 500)
    z[:4] = np.array([0, 1, 2 ** 64 - 1, 1 << 63], dtype=np.uint64)
    for party in (0, 1):
        for f in (0, 1, 16, 62):
            assert np.array_equal(oa.rescale(party, z, f), co.truncate_share(party, z, f))


def cache_of(plain, seed):
    """(F, [X_0, X_1]) of a plain pool: F = X - B, X_i = B_i + i F."""
    b = [u64(seed, 1 + i, *plain.shape) for i in (0, 1)]
    f = plain - b[0] - b[1]
    return f, [b[0], b[1] + f], b


def triple(left, b, seed, product):
    """Opened E, shares of A and of C = product(A, B) for a secret left operand."""
    a = [u64(seed, 11 + i, *left.shape) for i in (0, 1)]
    e = left - a[0] - a[1]
    c = product(a[0] + a[1], b[0] + b[1])
    c0 = u64(seed, 13, *c.shape)
    return e, a, [c0, c - c0]


def test_scores_and_values_reconstruct_the_products():
    heads, kvh, d, page, kv = 4, 2, 6, 16, 19
    table = np.array([[1, 0]])
    q_start, kv_len = [0, 3], [kv]
    batch = list(oa.rows(q_start, kv_len, heads))
    pool = u64(901, 50, 2, page, kvh, 8)
    f, x, b = cache_of(pool, 902)
    gather = lambda p, h: oa.cached(p, table, 0, kv, h // 2, d)
    q = u64(901, 51, 3, heads, d)
    by_keys = lambda l, p: np.stack([[gather(p, h) @ l[t, h] for h in range(heads)] for t in range(3)])
    e, a, c = triple(q, b, 903, by_keys)
    zero = np.zeros((3, heads, kv), dtype=np.uint64)
    z = [oa.scores(i, batch, e, a[i], f, x[i], table, c[i], 0, None, zero) for i in (0, 1)]
    want = by_keys(q, pool)
    for _, t, h, v in batch:
        assert v == kv - 2 + t
        assert np.array_equal((z[0] + z[1])[t, h, :v], want[t, h, :v])
        assert not z[0][t, h, v:].any()
    w = u64(901, 52, 3, heads, kv)
    seen = np.zeros((3, heads, kv), dtype=np.uint64)
    for _, t, h, v in batch:
        seen[t, h, :v] = 1
    by_rows = lambda l, p: np.stack([[(l[t, h] * seen[t, h]) @ gather(p, h) for h in range(heads)] for t in range(3)])
    e, a, c = triple(w, b, 904, by_rows)
    zero = np.zeros((3, heads, d), dtype=np.uint64)
    z = [oa.values(i, batch, e, a[i], f, x[i], table, c[i], 0, None, zero) for i in (0, 1)]
    assert np.array_equal(z[0] + z[1], by_rows(w, pool))


def test_weights_reconstruct_the_squares_and_their_sums():
    batch = [(0, 0, 0, 7), (0, 0, 1, 0), (0, 1, 0, 9), (0, 1, 1, 3)]
    s = u64(905, 1, 2, 2, 9) >> U(36)
    r = [u64(905, 2 + i, 2, 2, 9) for i in (0, 1)]
    square = (r[0] + r[1]) * (r[0] + r[1])
    r2 = [u64(905, 4, 2, 2, 9)]
    r2.append(square - r2[0])
    d_0 = u64(905, 5, 2, 2, 9)
    d_1 = s - r[0] - r[1] - d_0
    zero, none = np.zeros((2, 2, 9), dtype=np.uint64), np.zeros((2, 2), dtype=np.uint64)
    got = [oa.weights(i, batch, d_0, d_1, r[i], r2[i], 12345, 0, None, zero, none) for i in (0, 1)]
    want = (s + U(12345)) ** U(2)
    for _, t, h, v in batch:
        assert np.array_equal((got[0][0] + got[1][0])[t, h, :v], want[t, h, :v])
        assert (got[0][1] + got[1][1])[t, h] == np.add.reduce(want[t, h, :v], dtype=np.uint64)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_reconstructs_the_rotated_vector(interleaved):
    """Every rescaling of a shared value is off by less than one unit (2^-16).  A rotated word adds two of the first,
    each times at most one, its own, and the tables' roundings (2^-17 each) times the two words: less than
    2^-16 (1 + 1 + 1) + 2^-17 (|x_p| + |x_q|)."""
    t, heads, d, rot = 3, 2, 10, 8
    x = rng.gaussian_f64(906, 1, t * heads * d).reshape(t, heads * d)
    pos = np.array([0, 5, 4095])
    angle = np.arange(4096)[:, None] * 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    fixed = lambda v: np.round(v * 65536).astype(np.int64).view(np.uint64)
    big = np.round(x * 2.0 ** 32).astype(np.int64).view(np.uint64)
    first = u64(906, 2, t, heads * d)
    y = [oa.rotate(i, s, pos, fixed(np.cos(angle)), fixed(np.sin(angle)), heads, 16, 16, None, interleaved)
         for i, s in enumerate((first, big - first))]
    got = signed(y[0] + y[1]).reshape(t, heads, d) / 65536.0
    xs = x.reshape(t, heads, d)
    want, bound = xs.copy(), np.full(xs.shape, 2.0 ** -16)
    for j in range(rot // 2):
        p, q = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, s = np.cos(angle[pos, j])[:, None], np.sin(angle[pos, j])[:, None]
        want[:, :, p] = xs[:, :, p] * c - xs[:, :, q] * s
        want[:, :, q] = xs[:, :, q] * c + xs[:, :, p] * s
        b = 3 * 2.0 ** -16 + 2.0 ** -17 * (np.abs(xs[:, :, p]) + np.abs(xs[:, :, q]) + 2.0 ** -15)
        bound[:, :, p] = bound[:, :, q] = b
    assert (np.abs(got - want) <= bound + 2.0 ** -32).all()


def test_cache_rows_reconstruct_the_cached_values():
    d = [u64(907, 1 + i, 4, 5) for i in (0, 1)]
    b = [u64(907, 3 + i, 4, 5) for i in (0, 1)]
    pools = [u64(907, 5 + i, 6, 5) for i in (0, 1)]
    slots = [3, -1, 0, 6]
    f, x = zip(*[oa.cache_write(i, d[0], d[1], b[i], slots, pools[0], pools[1]) for i in (0, 1)])
    plain = d[0] + d[1] + b[0] + b[1]
    assert np.array_equal(f[0], f[1])
    for t in (0, 2):
        assert np.array_equal((x[0] + x[1])[slots[t]], plain[t])
    assert np.array_equal(f[0][[1, 2, 4, 5]], pools[0][[1, 2, 4, 5]])
    keep = u64(907, 9, 4, 5)
    e, a = zip(*[oa.cache_read(i, f[i], x[i], slots, keep, keep) for i in (0, 1)])
    for t in (0, 2):
        assert np.array_equal(e[0][t] + a[0][t] + a[1][t], plain[t])
        assert np.array_equal(a[0][t], b[0][t]) and np.array_equal(a[1][t], b[1][t])
    assert np.array_equal(e[0][[1, 3]], keep[[1, 3]])


def test_batch_struct_matches_the_header():
    from paper_2505_07239_amd import binding
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "comet_ring.h")).read(), flags=re.S)
    body = re.search(r"typedef struct comet_kv_batch \{(.*?)\} comet_kv_batch;", text, flags=re.S).group(1)
    names, pointers = [], []
    for field in body.split(";"):
        for name in re.sub(r"\s+", " ", field).strip().split(","):
            if name.strip():
                names.append(name.split()[-1].lstrip("*"))
                pointers.append("*" in name)
    assert names == [n for n, _ in binding._Batch._fields_]
    assert pointers == [c is ctypes.c_void_p for _, c in binding._Batch._fields_]
    assert ctypes.sizeof(binding._Batch) == 8 * 4 + 4 * ctypes.sizeof(ctypes.c_void_p)


def test_null_context_and_tensors_off_the_gpu_are_refused():
    torch = pytest.importorskip("torch")
    import paper_2505_07239_amd as comet
    lib = comet.load_library()
    batch = comet.binding._Batch()
    assert lib.comet_cache_write(None, 0, None, None, None, None, 1, 1, None, None, 1) == -1
    assert lib.comet_cache_read(None, 0, None, None, None, 1, 1, 1, None, None) == -1
    assert lib.comet_rotate_share(None, 0, None, 4, None, None, None, 1, 1, 1, 4, 4, 0, 0, 16, None, None) == -1
    for call in (lib.comet_attention_scores, lib.comet_attention_values):
        assert call(None, 0, ctypes.byref(batch), 2, 2, 1, 2, 0, *[None] * 8, 0) == -1
    assert lib.comet_attention_weights(None, 0, ctypes.byref(batch), 2, 0, 0, *[None] * 7) == -1
    cpu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        comet.KVBatch(1, 1, 1, cpu, cpu[:1], cpu[None, :], 16, 1)
