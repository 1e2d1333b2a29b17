"""The serving operators through the C ABI against their float64 definitions (oracle/serve_oracle.py).

Bounds count roundings.  u = 2^-24 is fp32's, 2^-8 bf16's half step relative to a value; a sum of n terms is off by at most n u times
the sum of their sizes."""
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def B():
    from paper_2603_03251_amd import binding
    return binding


def f64(t):
    return t.double().cpu().numpy()


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).cuda().contiguous()


def randn(g, shape, dtype):
    return torch.randn(shape, generator=g).to(dtype).cuda()


def gen(seed):
    return torch.Generator().manual_seed(seed)


SCALINGS = {"plain": dict(), "linear": dict(factor=4.0), "bands": dict(factor=32.0, low=1.0, high=4.0, original=8192.0),
            "ramp": dict(factor=16.0, low=1.0, high=32.0, original=8192.0)}


def _rope(B, theta, rot, layout, scaling, magnitude=1.0):
    return (B.rope_config(theta, rot, layout=layout, scaling=scaling, magnitude=magnitude, **SCALINGS[scaling]),
            S.rope_frequencies(theta, rot, scaling, **SCALINGS[scaling]))


def check_rotated(got, x, positions, freq, layout, magnitude, dtype):
    """cos and sin: the angle is rounded once (below 1) and the series evaluated in fp32, 4 u of 1; the products and their sum 3 u more, the
    magnitude 1: 8 u (|a| + |b|).  Before that the angle, of fp64 numbers: a frequency carries 2^-52 from its exponent's rounding times at most
    that exponent (f times which stays below 1), the product another 2^-53: 2^-50 per position.  Then one rounding to the result's type."""
    want, size = S.rotate(f64(x), np.asarray(positions, np.float64), freq, layout, magnitude)
    pos = np.abs(np.asarray(positions, np.float64))[..., None, None]
    bound = size * (8 * U + pos * 2.0 ** -50) + np.abs(want) * HALF[dtype]
    rot = 2 * len(freq)
    err = np.abs(f64(got) - want)
    assert np.all(err <= bound), float((err / np.maximum(bound, 1e-300)).max())
    assert np.array_equal(f64(got)[..., rot:], f64(x.to(dtype))[..., rot:])        # what is not rotated passes as it is


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,D,rot,layout,scaling", [
    (4, 64, 64, "half", "plain"), (40, 64, 64, "half", "bands"), (72, 128, 128, "half", "ramp"), (1, 128, 128, "interleaved", "linear"),
    (9, 128, 96, "interleaved", "ramp"), (5, 64, 2, "half", "plain"), (3, 64, 2, "interleaved", "plain"), (33, 128, 64, "half", "bands"),
    (7, 64, 48, "half", "linear"), (8, 128, 124, "half", "plain")])
def test_rope(B, dtype, heads, D, rot, layout, scaling):
    g = gen(heads + rot)
    cfg, freq = _rope(B, 500000.0, rot, layout, scaling, 1.25)
    for positions in ([0], [1], [-7, 0, 5], [8191, 131072, 2147483647, -2147483648], list(range(1000, 1000 + 203))):
        x = randn(g, (len(positions), heads, D), dtype)
        out = torch.full_like(x, 7.0)
        B.ssd_rope(cfg, x, i32(positions), out)
        check_rotated(out, x, positions, freq, layout, 1.25, dtype)


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_large_calls_give_the_bits_of_small_ones(B, dtype, cache, layout):
    """170 MB and more in a call, against calls of 700 rows; in place too."""
    cfg, _ = _rope(B, 500000.0, 96, layout, "bands")
    g, T, hq, hkv, D, page = gen(5), 4099 if dtype == BF16 else 2111, 64, 8, 128, 32
    blocks = -(-T // page)
    q, k, v = randn(g, (1, T, hq, D), dtype), randn(g, (1, T, hkv, D), dtype), randn(g, (1, T, hkv, D), dtype)
    pos, table = i32(np.arange(T)[None] + 100000), i32(np.random.default_rng(1).permutation(blocks)[None])
    slots = i32(np.arange(T)[None])
    results = []
    for step in (T, 700):
        pools = [torch.full((blocks, page, hkv, D), -1.0, dtype=cache, device="cuda") for _ in range(2)]
        kv, out = B.paged_kv(pools[0], pools[1], table), torch.zeros_like(q)
        for i in range(0, T, step):
            part = slice(i, min(i + step, T))
            B.ssd_rope_append(cfg, q[:, part], k[:, part], v[:, part], pos[:, part].contiguous(), kv, out[:, part], slots=slots[:, part].contiguous())
        results.append((out, *pools))
    assert all(torch.equal(x, y) for x, y in zip(*results))
    B.ssd_rope(cfg, q[0], pos[0], q[0])
    assert torch.equal(q, results[0][0])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_of_views_and_in_place(B, dtype, layout):
    """Rows behind others' elements, at offsets and strides of one element; in place."""
    cfg, freq = _rope(B, 10000.0, 64, layout, "plain")
    g = gen(3)
    pos = [3, 900, 17]
    for ld, offset in ((1024, 0), (1000, 8), (901, 3), (902, 1)):
        store = randn(g, (3 * ld + 16,), dtype)
        before = store.clone()
        x = torch.as_strided(store, (3, 6, 128), (ld, 128, 1), offset)
        was = x.clone()
        out = torch.zeros((3, 6, 128), dtype=dtype, device="cuda")
        B.ssd_rope(cfg, x, i32(pos), out)
        check_rotated(out, was, pos, freq, layout, 1.0, dtype)
        assert torch.equal(store, before)
        B.ssd_rope(cfg, x, i32(pos), x)
        assert torch.equal(x, out)
        x.copy_(was)
        assert torch.equal(store, before)             # nothing between the rows was written
    B.ssd_rope(cfg, torch.empty((0, 6, 128), dtype=dtype, device="cuda"), i32([]), torch.empty((0, 6, 128), dtype=dtype, device="cuda"))


class Cache:
    """A pool of pages filled with NaN, pages dealt in a shuffled order; entries of positions that nothing holds are garbage."""

    def __init__(self, B, g, nb, blocks, page, hkv, D, dtype, mapped=None, together=False, spare=3):
        n = nb * blocks + spare
        if together:                                  # keys and values of a page one behind the other
            both = torch.full((n, 2, page, hkv, D), float("nan"), dtype=dtype).cuda()
            self.k, self.v = both[:, 0], both[:, 1]
        else:
            self.k = torch.full((n, page, hkv, D), float("nan"), dtype=dtype).cuda()
            self.v = torch.full((n, page, hkv, D), float("nan"), dtype=dtype).cuda()
        order = torch.randperm(n, generator=g).numpy()
        self.table = order[:nb * blocks].reshape(nb, blocks).astype(np.int32)
        if mapped is not None:
            for b in range(nb):
                self.table[b, mapped[b]:] = np.random.default_rng(b).choice([-1, -2 ** 31, n, 2 ** 31 - 1, 2 ** 24], blocks - mapped[b])
        self.n, self.page = n, page
        self.dev_table = i32(self.table)
        self.kv = B.paged_kv(self.k, self.v, self.dev_table)

    def place(self, b, slot):
        return S.place(self.table, self.n, self.page, b, slot)

    def set_table(self, table):
        self.table = table
        self.dev_table.copy_(i32(table))


@pytest.mark.parametrize("dtype,cache", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("hq,hkv,D,rot,layout,page,T,together", [
    (4, 4, 64, 64, "half", 32, 1, False), (32, 8, 64, 64, "half", 8, 6, True), (64, 8, 128, 128, "half", 32, 17, False),
    (8, 1, 128, 64, "interleaved", 1024, 40, False), (6, 2, 64, 20, "half", 16, 5, True), (16, 16, 128, 128, "interleaved", 64, 131, True)])
def test_append(B, dtype, cache, hq, hkv, D, rot, layout, page, T, together):
    nb, g = 3, gen(T)
    blocks = 2 + (T + 60) // page
    c = Cache(B, g, nb, blocks, page, hkv, D, cache, together=together)
    table = c.table.copy()
    table[1, 0] = -1                                   # a page that sequence 1 has given back
    c.set_table(table)
    cfg, freq = _rope(B, 500000.0, rot, layout, "bands", 0.5)
    qkv = randn(g, (nb, T, (hq + 2 * hkv) * D), dtype)
    q, k, v = (t.unflatten(2, (h, D)) for t, h in zip(qkv.split([hq * D, hkv * D, hkv * D], dim=2), (hq, hkv, hkv)))
    positions = np.array([[50 + t, 5 + t, 90000 + t] for t in range(T)]).T
    slots = np.array([[50 + t, 5 + t, T - 1 - t] for t in range(T)]).T
    slots[0, T // 2] = -1
    if T > 2:
        slots[2, 0] = blocks * page                    # behind the table
        slots[2, 1] = 2 ** 31 - 1
    k0, v0 = f64(c.k), f64(c.v)
    out = torch.full((nb, T, hq, D), 7.0, dtype=dtype, device="cuda")
    B.ssd_rope_append(cfg, q, k, v, i32(positions), c.kv, out, slots=i32(slots))
    check_rotated(out, q, positions, freq, layout, 0.5, dtype)
    want_k, size = S.rotate(f64(k), positions, freq, layout, 0.5)
    got_k, got_v = f64(c.k), f64(c.v)
    stored = 0
    for b in range(nb):
        for t in range(T):
            at = c.place(b, int(slots[b, t]))
            if at is None:
                continue
            stored += 1
            bound = size[b, t] * (8 * U + positions[b, t] * 2.0 ** -50) + np.abs(want_k[b, t]) * HALF[cache]
            assert np.all(np.abs(got_k[at] - want_k[b, t]) <= bound)
            assert np.array_equal(got_v[at], f64(v[b, t].to(cache)))
            got_k[at], got_v[at] = k0[at], v0[at]
    assert stored >= T
    assert np.array_equal(got_k, k0, equal_nan=True) and np.array_equal(got_v, v0, equal_nan=True)   # and nothing else was written
    # without slots a row goes to its position; the queries in place
    if positions[:2].max() < blocks * page:
        again = Cache(B, gen(T), nb, blocks, page, hkv, D, cache, together=together)
        B.ssd_rope_append(cfg, q, k, v, i32(positions), again.kv, q)
        assert torch.equal(q, out)
        assert torch.equal(again.k[again.place(0, 50)].float(), c.k[c.place(0, 50)].float()) or T // 2 == 0


def check_attention(B, c, q, visible, tail=None, scale=None, max_visible=None, with_lse=True, stream=None):
    """Scores: products of D terms, D + 2 roundings of scale sum |q k|, in powers of two one more of their size, and the exponential's 2 u;
    a weight is off by twice that (its sum's too), its planes by 2^-17 with bf16 queries (two of 8 bits) and 2^-24 with fp32 ones, sums of n
    weights and values by n u each; then one rounding to the result's type."""
    nb, T, hq, D = q.shape
    dtype, cache = q.dtype, c.k.dtype
    scale = D ** -0.5 if scale is None else scale
    visible = np.asarray(visible)
    most = int(visible.max()) if max_visible is None else max_visible
    most = max(most, 0)
    ws = torch.full((B.ssd_paged_attention_workspace_bytes(c.kv, nb, T, hq, most) // 4,), float("nan"), device="cuda")
    out = torch.full_like(q, float("nan"))
    lse = torch.full((nb, T, hq), float("nan"), device="cuda") if with_lse else None
    tails = None if tail is None else B.tail_kv(*tail)
    B.ssd_paged_attention(c.kv, q, i32(visible), most, out, ws, scale=scale, tail=tails, lse=lse, stream=stream)
    torch.cuda.synchronize()
    k, v, qh, got = f64(c.k), f64(c.v), f64(q), f64(out)
    tk, tv = (None, None) if tail is None else (f64(tail[0]), f64(tail[1]))
    worst = 0.0
    for b in range(nb):
        for t in range(T):
            at = [c.place(b, j) for j in range(min(max(int(visible[b, t]), 0), most))]
            keys, values = [k[a] for a in at if a], [v[a] for a in at if a]
            if tail is not None:
                keys, values = keys + list(tk[b, t, :tail[2]]), values + list(tv[b, t, :tail[2]])
            want, size, want_lse, score = S.attend(qh[b, t], keys, values, scale)
            planes = 2.0 ** -17 if dtype == BF16 and cache == BF16 else U
            off = (D + 4) * U * score + 4 * U
            bound = size * (2 * off + 2 * planes + 2 * (len(keys) + 16) * U) + np.abs(want) * HALF[dtype]
            finite = np.isfinite(want)
            assert np.array_equal(np.isnan(got[b, t]), np.isnan(want)) and np.array_equal(got[b, t][~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)])
            if finite.any():
                err = np.abs(got[b, t][finite] - want[finite])
                assert np.all(err <= bound[finite]), (b, t, float((err / np.maximum(bound[finite], 1e-300)).max()))
                worst = max(worst, float((err / np.maximum(bound[finite], 1e-30)).max()))
            if with_lse:
                g = f64(lse[b, t])
                if not keys:
                    assert np.all(np.isneginf(g))
                elif np.isfinite(want_lse).all():
                    assert np.all(np.abs(g - want_lse) <= off + (len(keys) + 16) * U + np.abs(want_lse) * 4 * U)
    return out, worst


TYPES = [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("hq,hkv,D", [(4, 4, 64), (32, 8, 64), (8, 1, 128), (14, 2, 128)])
@pytest.mark.parametrize("T", [1, 5, 17])
def test_attention_lengths(B, dtype, cache, hq, hkv, D, T):
    """Rows of no, one and many positions, at the edges of pages, steps and splits, each row another number."""
    g = gen(hq * T + D)
    lens = [[0, 1, 7, 8, 9], [31, 32, 33, 15, 16, 17], [127, 128, 129, 255, 256, 257, 300, 2]]
    for page in (8, 32, 128):
        blocks = -(-300 // page)
        visible = np.array([[row[t % len(row)] for t in range(T)] for row in lens])
        if T == 1:
            visible = np.array([[0], [33], [300]]) if page != 8 else np.array([[1], [129], [256]])
        c = Cache(B, g, 3, blocks, page, hkv, D, cache, mapped=[-(-max(int(r.max()), 0) // page) for r in visible], together=page == 32)
        for b in range(3):
            for j in range(int(visible[b].max())):
                c.k[c.place(b, j)] = randn(g, (hkv, D), cache)
                c.v[c.place(b, j)] = randn(g, (hkv, D), cache)
        check_attention(B, c, randn(g, (3, T, hq, D), dtype), visible, max_visible=300)


def _full_cache(B, g, nb, n, page, hkv, D, cache, **kw):
    c = Cache(B, g, nb, -(-n // page), page, hkv, D, cache, **kw)
    c.k.copy_(randn(g, tuple(c.k.shape), cache))
    c.v.copy_(randn(g, tuple(c.v.shape), cache))
    return c


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("hq,hkv,D,T,n", [(32, 8, 64, 1, 5000), (16, 2, 128, 3, 9001), (4, 4, 64, 24, 2100), (8, 1, 128, 40, 1500)])
def test_attention_over_long_caches(B, dtype, cache, hq, hkv, D, T, n):
    g = gen(n)
    c = _full_cache(B, g, 1, n, 32, hkv, D, cache)
    visible = np.arange(n - T + 1, n + 1)[None]
    q = randn(g, (1, T, hq, D), dtype)
    out, worst = check_attention(B, c, q, visible)
    again, _ = check_attention(B, c, q, visible, with_lse=False)
    assert torch.equal(out, again)                    # no order that changes


@pytest.mark.parametrize("dtype,cache,page", [(BF16, BF16, 32), (BF16, BF16, 8), (F32, BF16, 64), (F32, F32, 16), (F32, F32, 8), (BF16, F32, 128)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_over_caches_larger_than_the_memory_side_one(B, dtype, cache, page, D):
    """max_visible sizes the launch: with a bound for which the caches' lines are not kept, rows of few positions and none, garbage behind them."""
    g, nb, hq, hkv = gen(page + D), 6, 16, 8
    n = 200_000_000 // (nb * hkv * D * 2 * (2 if cache == BF16 else 4)) // page * page
    blocks = n // page
    lens = [0, 1, 700, 33, 256, 3000]
    c = Cache(B, g, nb, 3000 // page + 1, page, hkv, D, cache)
    table = np.full((nb, blocks), 2 ** 30, np.int32)
    table[:, :c.table.shape[1]] = c.table
    for b, m in enumerate(lens):
        table[b, -(-m // page):] = -7
        for j in range(m):
            c.k[c.place(b, j)] = randn(g, (hkv, D), cache)
            c.v[c.place(b, j)] = randn(g, (hkv, D), cache)
    c.table, c.dev_table = table, i32(table)
    c.kv = B.paged_kv(c.k, c.v, c.dev_table)
    check_attention(B, c, randn(g, (nb, 1, hq, D), dtype), np.array(lens)[:, None], max_visible=n)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("nb,T,splits", [(9, 1, 3), (12, 1, 2), (5, 1, 3), (8, 1, 1)])
def test_attention_of_rows_that_leave_a_last_round_of_blocks(B, dtype, cache, nb, T, splits):
    """288, 384 and 160 blocks' worth of rows are split to fill the units, 256 are not."""
    g, hkv, D, n = gen(nb), 32, 64, 2100
    c = _full_cache(B, g, nb, n, 32, hkv, D, cache)
    assert B.ssd_paged_attention_workspace_bytes(c.kv, nb, T, hkv, n) == nb * T * hkv * splits * (D + 2) * 4
    visible = np.array([[[n, 1, 768, 769, 0, 1536, 2099, 1537, 1024][b % 9]] * T for b in range(nb)])
    check_attention(B, c, randn(g, (nb, T, hkv, D), dtype), visible)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("length,capacity", [(0, 3), (1, 1), (5, 7), (70, 256)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_with_tails(B, dtype, cache, length, capacity, D):
    """Branches: rows that share a trunk up to a fork each, private keys behind it; rows with a tail alone."""
    g, nb, T, hq, hkv = gen(length), 2, 6, 8, 2
    c = _full_cache(B, g, nb, 400, 16, hkv, D, cache)
    tk, tv = (randn(g, (nb, T, capacity, hkv, D), cache) for _ in range(2))
    tk[:, :, length:] = float("nan")
    tv[:, :, length:] = float("inf")
    visible = np.array([[0, 1, 390, 391, 392, 17], [3, 2, 1, 0, 0, 40]])
    check_attention(B, c, randn(g, (nb, T, hq, D), dtype), visible, tail=(tk, tv, length))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(B, dtype, cache, D):
    """Infinities and NaN at positions that some rows of a block see and others do not, in keys and values, behind the last one, and in pages
    that are not the sequence's; pages missing in the middle."""
    g, nb, T, hq, hkv, n = gen(5), 2, 4, 8, 2, 200
    c = _full_cache(B, g, nb, n, 8, hkv, D, cache)
    table = c.table.copy()
    table[0, 3], table[0, 4], table[1, 0], table[1, 24] = -1, c.n, 2 ** 31 - 1, -2 ** 31
    c.set_table(table)
    visible = np.array([[150, 151, 152, 153], [200, 193, 199, 192]])
    c.v[c.place(0, 150)][0, 3] = float("inf")
    c.v[c.place(0, 151)][1, D - 1] = float("-inf")
    c.v[c.place(0, 152)][0, 5] = float("nan")
    c.k[c.place(0, 152)][1, 0] = float("nan")
    for j in range(153, 200):
        if c.place(0, j):
            c.v[c.place(0, j)] = float("nan")
            c.k[c.place(0, j)] = float("inf")
    out, _ = check_attention(B, c, randn(g, (nb, T, hq, D), dtype), visible, max_visible=200)
    assert torch.isfinite(out[0, 0]).all() and torch.isfinite(out[1]).all()
    assert not torch.isfinite(out[0, 1]).all() and not torch.isfinite(out[0, 3]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_blocks_of_two_tiles(B, D):
    """Enough rows that a block takes two tiles of them, each row another count of positions; rows whose last positions hold infinities and NaN that
    the row before does not see; an odd number of tiles; with tails."""
    g, nb, T, hq, hkv, n = gen(17), 3, 37, 64, 16, 330
    c = _full_cache(B, g, nb, n, 16, hkv, D, BF16)
    visible = np.random.default_rng(3).integers(0, n + 1, (nb, T))
    visible[0] = np.arange(n - T + 1, n + 1)
    visible[1, :4] = [0, 1, 256, 257]
    q = randn(g, (nb, T, hq, D), BF16)
    check_attention(B, c, q, visible, max_visible=n)
    for j in range(n - 6, n):
        c.v[c.place(0, j)][j % hkv, j % D] = float("inf") if j % 2 else float("nan")
    visible[1:] = np.minimum(visible[1:], 40)
    check_attention(B, c, q, visible, max_visible=n)
    tk, tv = (randn(g, (nb, T, 3, hkv, D), BF16) for _ in range(2))
    check_attention(B, c, q, np.minimum(visible, n - 6), tail=(tk, tv, 2), max_visible=n)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("nb,T,hq,hkv,D,page,n", [(1, 1, 64, 1, 128, 1024, 1500), (1, 70, 48, 1, 64, 32, 90), (130, 1, 2, 2, 64, 64, 70),
                                                  (2, 3, 5, 5, 128, 256, 400)])
def test_other_shapes(B, dtype, cache, nb, T, hq, hkv, D, page, n):
    """Many heads of one KV head, many rows, many sequences, pages larger than a step of all wavefronts."""
    g = gen(nb + T)
    c = _full_cache(B, g, nb, n, page, hkv, D, cache)
    check_attention(B, c, randn(g, (nb, T, hq, D), dtype), np.random.default_rng(nb).integers(0, n + 1, (nb, T)), max_visible=n)


def test_calls_on_two_streams_and_shared_pages(B):
    """Calls that overlap on two streams with a workspace each give the bits of calls one after the other; two sequences with the same pages; in
    place."""
    g = gen(31)
    c = _full_cache(B, g, 2, 2000, 32, 4, 128, BF16)
    table = c.table.copy()
    table[1, :40] = table[0, :40]
    c.set_table(table)
    qs = [randn(g, (2, 5, 16, 128), BF16) for _ in range(2)]
    vis = np.array([[1996, 1997, 1998, 1999, 2000], [1280, 1281, 1400, 700, 1]])
    want = [check_attention(B, c, q, vis)[0] for q in qs]
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(q) for q in qs]
    n = B.ssd_paged_attention_workspace_bytes(c.kv, 2, 5, 16, 2000)
    ws, v = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)], i32(vis)
    torch.cuda.synchronize()
    for _ in range(20):
        for s, q, o, w in zip(streams, qs, outs, ws):
            B.ssd_paged_attention(c.kv, q, v, 2000, o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    for most in (2000, 200):                             # split and joined, and in one launch
        q, o = qs[0].clone(), torch.empty_like(qs[0])
        B.ssd_paged_attention(c.kv, q, v, most, o, ws[0])
        B.ssd_paged_attention(c.kv, q, v, most, q, ws[0])
        assert torch.equal(q, o)


def test_rows_that_see_nothing(B):
    """Empty slots of a batch, negative counts, tables without a page: zeros, and -inf as the log of the sum; a bound of 0."""
    g = gen(9)
    for dtype, cache in TYPES:
        c = Cache(B, g, 3, 4, 16, 2, 64, cache)
        c.set_table(np.full((3, 4), -1, np.int32))
        q = randn(g, (3, 2, 4, 64), dtype)
        for visible, most in (([[0, 0], [0, 0], [0, 0]], 0), ([[-5, 0], [64, 3], [1, -2 ** 31]], 64)):
            out, _ = check_attention(B, c, q, visible, max_visible=most)
            assert torch.equal(out, torch.zeros_like(out))


def test_attention_clamps_to_the_bound_and_takes_other_scales(B):
    g = gen(11)
    c = _full_cache(B, g, 2, 96, 32, 2, 64, BF16)
    q = randn(g, (2, 3, 4, 64), BF16)
    check_attention(B, c, q, [[96, 2 ** 31 - 1, 40], [50, 51, 52]], max_visible=50)
    check_attention(B, c, q, [[96, 95, 94], [3, 2, 1]], scale=0.0)
    check_attention(B, c, q, [[96, 95, 94], [3, 2, 1]], scale=-0.3)


def test_attention_of_strided_queries(B):
    """Queries and outputs as parts of larger rows."""
    g = gen(12)
    c = _full_cache(B, g, 2, 96, 32, 2, 128, BF16)
    both = randn(g, (2, 3, 12, 128), BF16)
    q = both[:, :, 4:8]
    assert not q.is_contiguous()
    want, _ = check_attention(B, c, q.contiguous(), [[96, 95, 94], [3, 2, 1]])
    out = torch.zeros((2, 3, 12, 128), dtype=BF16, device="cuda")
    ws = torch.empty(B.ssd_paged_attention_workspace_bytes(c.kv, 2, 3, 4, 96), dtype=torch.uint8, device="cuda")
    B.ssd_paged_attention(c.kv, q, i32([[96, 95, 94], [3, 2, 1]]), 96, out[:, :, 8:], ws)
    assert torch.equal(out[:, :, 8:], want) and not out[:, :, :8].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_behind_32_bits(B, dtype):
    """A pool of more than 2^32 elements whose used pages are its last and first ones."""
    g, hq, hkv, D, page = gen(13), 8, 2, 128, 64
    stride = 1 << 24
    n = 258
    k = torch.empty((n * stride,), dtype=dtype, device="cuda")
    v = torch.empty((n * stride,), dtype=dtype, device="cuda")
    c = Cache.__new__(Cache)
    c.k, c.v = (torch.as_strided(t, (n, page, hkv, D), (stride, hkv * D, D, 1)) for t in (k, v))
    c.n, c.page = n, page
    c.table = np.array([[257, 0, 256, 129]], np.int32)
    c.dev_table = i32(c.table)
    c.kv = B.paged_kv(c.k, c.v, c.dev_table)
    for p in (257, 0, 256, 129):
        c.k[p].copy_(randn(g, (page, hkv, D), dtype))
        c.v[p].copy_(randn(g, (page, hkv, D), dtype))
    cfg, freq = _rope(B, 10000.0, 128, "half", "plain")
    q, kk, vv = randn(g, (1, 2, hq, D), dtype), randn(g, (1, 2, hkv, D), dtype), randn(g, (1, 2, hkv, D), dtype)
    out = torch.empty_like(q)
    B.ssd_rope_append(cfg, q, kk, vv, i32([[60, 61]]), c.kv, out)
    assert torch.equal(c.v[257, 60:62], vv[0])
    want, _ = S.rotate(f64(kk), np.array([[60, 61]]), freq, "half")
    assert np.abs(f64(c.k[257, 60:62]) - want[0]).max() <= np.abs(want).max() * HALF[dtype] + 16 * U * 8
    small = Cache.__new__(Cache)                       # the same pages in a small pool, for the check
    order = [257, 0, 256, 129]
    small.k, small.v = (torch.stack([t[p] for p in order]) for t in (c.k, c.v))
    small.n, small.page, small.table = 4, page, np.array([[0, 1, 2, 3]], np.int32)
    small.dev_table = i32(small.table)
    small.kv = B.paged_kv(small.k, small.v, small.dev_table)
    want, _ = check_attention(B, small, out, [[255, 256]])
    ws = torch.empty(B.ssd_paged_attention_workspace_bytes(c.kv, 1, 2, hq, 256), dtype=torch.uint8, device="cuda")
    got = torch.empty_like(out)
    B.ssd_paged_attention(c.kv, out, i32([[255, 256]]), 256, got, ws)
    assert torch.equal(got, want)


def _verify(B, target, draft, spec, ua, ub, drafted=None, stream=None):
    nb, K = spec.shape
    V = target.shape[2]
    k = torch.full((nb,), -9, dtype=torch.int32, device="cuda")
    t = torch.full((nb,), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((B.ssd_verify_probs_workspace_bytes(nb, V) // 4,), float("nan"), device="cuda")
    dev = lambda a: None if a is None else torch.as_tensor(a, dtype=F32).cuda()
    B.ssd_verify_probs(dev(target), dev(draft), i32(spec), dev(ua), dev(ub), k, t, ws, drafted=None if drafted is None else i32(drafted), stream=stream)
    torch.cuda.synchronize()
    got = list(zip(k.tolist(), t.tolist()))
    want = [S.verify_probs(target[b], None if draft is None else draft[b], spec[b], ua[b], ub[b], None if drafted is None else drafted[b]) for b in range(nb)]
    assert got == want, [(b, g, w) for b, (g, w) in enumerate(zip(got, want)) if g != w][:5]
    return got


def _probs(g, shape, spread):
    z = g.standard_normal(shape) * spread
    p = np.exp(z - z.max(axis=-1, keepdims=True))
    return (p / p.sum(axis=-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("V", [2, 5, 255, 256, 257, 1000, 4099, 50257, 128256])
@pytest.mark.parametrize("nb,K", [(1, 1), (3, 5), (5, 15)])
def test_verify_probs(B, V, nb, K):
    g = np.random.default_rng(V + K)
    seen = set()
    for certain in (False, True):
        z = g.standard_normal((nb, K + 1, V)) * 2
        soft = lambda x: np.exp(x - x.max(axis=-1, keepdims=True)) / np.exp(x - x.max(axis=-1, keepdims=True)).sum(axis=-1, keepdims=True)
        p = soft(z + 0.3 * g.standard_normal(z.shape)).astype(np.float32)
        q = soft(z[:, :K] + 0.3 * g.standard_normal((nb, K, V)))
        spec = np.array([[g.choice(V, p=q[b, i]) for i in range(K)] for b in range(nb)])
        q = None if certain else q.astype(np.float32)
        ua, ub = g.random((nb, K)).astype(np.float32) * 0.999, g.random(nb).astype(np.float32) * 0.999
        if certain:
            ua *= p[np.arange(nb)[:, None], np.arange(K), spec] * 1.3       # or nothing would be accepted
        for drafted in (None, g.integers(0, K + 1, nb)):
            for got in _verify(B, p, q, spec, ua, ub, drafted):
                seen.add(got[0])
    assert len(seen) > 1 or K == 1


def test_verify_of_a_large_batch(B):
    g = np.random.default_rng(8)
    nb, K, V = 300, 3, 771
    p, q = _probs(g, (nb, K + 1, V), 1.0), _probs(g, (nb, K, V), 1.0)
    spec = q.argmax(axis=2)
    p[np.arange(nb)[:, None], np.arange(K), spec] *= 20
    got = _verify(B, p, q, spec, g.random((nb, K)).astype(np.float32), g.random(nb).astype(np.float32) * 0.999, g.integers(-2, K + 3, nb))
    assert {k for k, _ in got} == set(range(K + 1))


def test_verify_at_the_edges(B):
    """Random numbers of 0 and as near 1 as they come, and outside; u q = p exactly; masses of zero at both ends; nothing left of p - q; rows
    without mass; tokens outside the vocabulary; entries that are not finite."""
    V, K = 600, 3
    p = np.zeros((1, K + 1, V), np.float32)
    p[:, :, 10:590:7] = 1.0 / 83
    q = np.zeros((1, K, V), np.float32)
    q[:, :, 3:590:7] = 2.0 / 83
    q[:, :, 17] = 1.0 / 83
    near = np.float32(1.0 - 2.0 ** -24)
    for ub in (0.0, near, 1.0, 5.0, -1.0, np.nan, 0.5):
        for spec, ua in (([17, 17, 17], [0.0, 0.0, 0.0]), ([17, 17, 17], [near, near, near]), ([17, 17, 24], [0.5, 1.0, 0.5]), ([3, 3, 3], [0.0, 0.0, 0.0]),
                         ([17, -1, 17], [0.0, 0.0, 0.0]), ([V, 17, 17], [0.0, 0.0, 0.0]), ([2 ** 31 - 1, 0, 0], [0.0] * 3), ([10, -2 ** 31, 0], [0.0] * 3)):
            got = _verify(B, p, q, np.array([spec]), np.array([ua], np.float32), np.array([ub], np.float32))
            assert got[0][1] >= 0 and p[0, 0, got[0][1]] > 0
            _verify(B, p, None, np.array([spec]), np.array([ua], np.float32) * 0.02, np.array([ub], np.float32))
    # exactly p = u q: not accepted; one step less of u: accepted
    assert _verify(B, p, q, np.array([[17] * 3]), np.array([[1.0] * 3], np.float32), np.array([0.3], np.float32))[0][0] == 0
    assert _verify(B, p, q, np.array([[17] * 3]), np.array([[near] * 3], np.float32), np.array([0.3], np.float32))[0][0] == 3
    # the draft is the target: a rejection (of a token that neither holds) leaves nothing, and p itself decides
    assert _verify(B, p, p[:, :K].copy(), np.array([[0, 0, 0]]), np.zeros((1, K), np.float32), np.array([0.999], np.float32)) == [(0, 584)]
    # rows without mass
    zero = np.zeros_like(p)
    assert _verify(B, zero, q, np.array([[17] * 3]), np.zeros((1, K), np.float32), np.array([0.5], np.float32)) == [(0, -1)]
    assert _verify(B, zero, None, np.array([[17] * 3]), np.zeros((1, K), np.float32), np.array([0.5], np.float32), [0]) == [(0, -1)]
    # what is not finite or not positive counts for nothing
    odd = p.copy()
    odd[:, :, 10], odd[:, :, 24], odd[:, :, 31], odd[:, :, 38] = np.nan, np.inf, -1.0, -np.inf
    bad_q = q.copy()
    bad_q[:, :, 45], bad_q[:, :, 52] = np.nan, np.inf
    for ub in (0.0, 0.01, 0.5, near):
        got = _verify(B, odd, bad_q, np.array([[10, 17, 17]]), np.zeros((1, K), np.float32), np.array([ub], np.float32))
        assert got[0][0] == 0 and got[0][1] not in (10, 24, 31, 38, 45, 52)
        _verify(B, odd, None, np.array([[17, 24, 17]]), np.zeros((1, K), np.float32), np.array([ub], np.float32))


def test_verify_takes_rows_apart(B):
    """Rows behind one another's padding, on 16 bytes and not, through the C entry (NaN in the padding)."""
    g = np.random.default_rng(4)
    nb, K, V = 2, 4, 1001
    p, q = _probs(g, (nb, K + 1, V), 2.0), _probs(g, (nb, K, V), 2.0)
    spec = p[:, :K].argmax(axis=2)
    ua, ub = g.random((nb, K)).astype(np.float32), g.random(nb).astype(np.float32)
    want = [S.verify_probs(p[b], q[b], spec[b], ua[b], ub[b]) for b in range(nb)]
    for p_ld, q_ld, skip in ((1004, 1008, 0), (1001, 1003, 0), (1004, 1004, 1)):
        sp = torch.full((nb * (K + 1) * p_ld + 4,), float("nan"), device="cuda")
        sq = torch.full((nb * K * q_ld + 4,), float("nan"), device="cuda")
        torch.as_strided(sp, (nb, K + 1, V), ((K + 1) * p_ld, p_ld, 1), skip).copy_(torch.from_numpy(p))
        torch.as_strided(sq, (nb, K, V), (K * q_ld, q_ld, 1), skip).copy_(torch.from_numpy(q))
        k, t = (torch.zeros(nb, dtype=torch.int32, device="cuda") for _ in range(2))
        ws = torch.empty(B.ssd_verify_probs_workspace_bytes(nb, V), dtype=torch.uint8, device="cuda")
        keep = [i32(spec), torch.from_numpy(ua).cuda(), torch.from_numpy(ub).cuda()]
        B._check(B.lib.ssd_verify_probs(sp.data_ptr() + 4 * skip, p_ld, sq.data_ptr() + 4 * skip, q_ld, keep[0].data_ptr(), None, keep[1].data_ptr(),
                                        keep[2].data_ptr(), nb, K, V, k.data_ptr(), t.data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream))
        torch.cuda.synchronize()
        assert list(zip(k.tolist(), t.tolist())) == want


def test_the_binding_refuses_what_the_kernels_would_read_wrongly(B):
    g = gen(1)
    c = _full_cache(B, g, 2, 64, 32, 2, 64, BF16)
    q = randn(g, (2, 3, 4, 64), BF16)
    vis, ws = i32([[1, 2, 3]] * 2), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    cfg, _ = _rope(B, 10000.0, 64, "half", "plain")
    kk = randn(g, (2, 3, 2, 64), BF16)
    for bad in (lambda: B.ssd_paged_attention(c.kv, q.transpose(2, 3).contiguous().transpose(2, 3), vis, 64, q, ws),
                lambda: B.ssd_paged_attention(c.kv, q, vis.long(), 64, q, ws),
                lambda: B.ssd_paged_attention(c.kv, q, vis.cpu(), 64, q, ws),
                lambda: B.ssd_paged_attention(c.kv, q, vis[:1], 64, q, ws),
                lambda: B.ssd_paged_attention(c.kv, q, vis, 64, q.float(), ws),
                lambda: B.ssd_paged_attention(c.kv, q, vis, 64, q, ws[:64]),
                lambda: B.ssd_paged_attention(c.kv, torch.cat([q, q]), torch.cat([vis, vis]), 64, torch.cat([q, q]), ws),
                lambda: B.ssd_paged_attention(c.kv, q, vis, 64, q, ws, lse=torch.empty((2, 3), device="cuda")),
                lambda: B.ssd_paged_attention(c.kv, q, vis, 64, q, ws, tail=B.tail_kv(kk[:, :, None].float(), kk[:, :, None].float(), 1)),
                lambda: B.paged_kv(c.k, c.v.float(), c.dev_table), lambda: B.paged_kv(c.k, c.v, c.dev_table.long()),
                lambda: B.paged_kv(c.k[:, :, :, :32], c.v[:, :, :, :32], c.dev_table), lambda: B.paged_kv(c.k.cpu(), c.v.cpu(), c.dev_table),
                lambda: B.ssd_rope_append(cfg, q, kk.float(), kk, vis, c.kv, q), lambda: B.ssd_rope_append(cfg, q, kk, kk, vis[:, :2], c.kv, q),
                lambda: B.ssd_rope_append(cfg, q, kk[:, :, :1], kk[:, :, :1], vis, c.kv, q),
                lambda: B.ssd_rope(cfg, q[0], i32([1, 2]), q[0]), lambda: B.ssd_rope(cfg, q[0].half(), i32([1, 2, 3]), q[0].half()), lambda: B.ssd_rope(cfg, q[0], i32([1, 2, 3]), q[0].float()),
                lambda: B.ssd_rope(cfg, q[0].expand(3, 4, 64)[:, :1].expand(3, 4, 64), i32([1, 2, 3]), q[0])):
        with pytest.raises(ValueError):
            bad()


def _step_buffers(B, c, nb, T, hq, hkv, D, V, most):
    mk = lambda shape, dt: torch.zeros(shape, dtype=dt, device="cuda")
    return dict(qkv=mk((nb, T, (hq + 2 * hkv) * D), BF16), pos=mk((nb, T), torch.int32), vis=mk((nb, T), torch.int32), slots=mk((nb, T), torch.int32),
                q=mk((nb, T, hq, D), BF16), out=mk((nb, T, hq, D), BF16), k=mk((nb,), torch.int32), t=mk((nb,), torch.int32),
                w=mk((hq * D, V), F32), draft=mk((nb, T - 1, V), F32), spec=mk((nb, T - 1), torch.int32), ua=mk((nb, T - 1), F32), ub=mk((nb,), F32),
                probs=mk((nb, T, V), F32),
                ws=torch.empty(B.ssd_paged_attention_workspace_bytes(c.kv, nb, T, hq, most), dtype=torch.uint8, device="cuda"),
                ws2=torch.empty(B.ssd_verify_probs_workspace_bytes(nb, V), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("side", [False, True])
def test_steps_of_a_target(B, captured, side):
    """Rounds of a one-layer target: projections, rotary positions and append, attention, a head, verification of K drafted tokens; accepted
    tokens stay in the cache, rejected ones are written over by the next round.  Eagerly, and as one captured graph that is replayed with
    new inputs and the eager work between; on the default stream, and on another."""
    nb, K, hq, hkv, D, V, page, most = 3, 4, 8, 2, 64, 333, 16, 128
    T, g, cpu = K + 1, gen(21), np.random.default_rng(21)
    c = Cache(B, g, nb, most // page, page, hkv, D, BF16)
    s = _step_buffers(B, c, nb, T, hq, hkv, D, V, most)
    s["w"].copy_(torch.randn(s["w"].shape, generator=g) * 0.3)
    cfg, freq = _rope(B, 10000.0, 32, "interleaved", "bands")
    lens = np.array([0, 13, 40])
    prompt = torch.randn((nb, 40, 2, hkv, D), generator=g).to(BF16)
    for b in range(nb):
        for j in range(lens[b]):
            c.k[c.place(b, j)], c.v[c.place(b, j)] = prompt[b, j, 0].cuda(), prompt[b, j, 1].cuda()
    heads = s["qkv"].split([hq * D, hkv * D, hkv * D], dim=2)
    qh, kh, vh = (t.unflatten(2, (h, D)) for t, h in zip(heads, (hq, hkv, hkv)))

    def step():
        B.ssd_rope_append(cfg, qh, kh, vh, s["pos"], c.kv, s["q"], slots=s["slots"])
        B.ssd_paged_attention(c.kv, s["q"], s["vis"], most, s["out"], s["ws"])
        torch.softmax(torch.mm(s["out"].reshape(nb * T, hq * D).float(), s["w"]), dim=1, out=s["probs"].view(nb * T, V))
        B.ssd_verify_probs(s["probs"], s["draft"], s["spec"], s["ua"], s["ub"], s["k"], s["t"], s["ws2"])

    stream = torch.cuda.Stream() if side else torch.cuda.current_stream()
    torch.cuda.synchronize()
    graph = None
    accepted = []
    with torch.cuda.stream(stream):
        for rnd in range(5):
            s["qkv"].copy_(torch.randn(s["qkv"].shape, generator=g))
            pos = lens[:, None] + np.arange(T)
            s["pos"].copy_(i32(pos)); s["slots"].copy_(i32(pos)); s["vis"].copy_(i32(pos + 1))
            before_k, before_v = c.k.clone(), c.v.clone()
            z = torch.randn((nb, K, V), generator=g)
            s["draft"].copy_(torch.softmax(z, dim=2))
            s["spec"].copy_(torch.randint(0, V, (nb, K), generator=g))
            s["ua"].copy_(torch.rand((nb, K), generator=g)); s["ub"].copy_(torch.rand((nb,), generator=g) * 0.999)
            if captured and graph is None:
                step()                                        # libraries load before the capture
                torch.cuda.synchronize()
                c.k.copy_(before_k); c.v.copy_(before_v)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream if side else None):
                    step()
            graph.replay() if captured else step()
            torch.cuda.synchronize()
            got = {n: t.clone() for n, t in s.items() if n in ("q", "out", "probs", "k", "t")}
            cache = c.k.clone(), c.v.clone()
            # the definitions, from the library's own input of each operator
            check_rotated(got["q"], qh, pos, freq, "interleaved", 1.0, BF16)
            want_k, size = S.rotate(f64(kh), pos, freq, "interleaved")
            for b in range(nb):
                for t in range(T):
                    at = c.place(b, int(pos[b, t]))
                    assert np.all(np.abs(f64(c.k[at]) - want_k[b, t]) <= size[b, t] * 9 * U + np.abs(want_k[b, t]) * HALF[BF16])
                    assert torch.equal(c.v[at], vh[b, t])
            out, _ = check_attention(B, c, got["q"], pos + 1, max_visible=most)
            assert torch.equal(out, got["out"])
            p, q = got["probs"].cpu().numpy(), s["draft"].cpu().numpy()
            for b in range(nb):
                k, t = S.verify_probs(p[b], q[b], s["spec"][b].cpu().numpy(), s["ua"][b].cpu().numpy(), float(s["ub"][b]))
                assert (k, t) == (int(got["k"][b]), int(got["t"][b]))
            accepted += got["k"].tolist()
            if captured:                                      # the eager calls give the same bits
                c.k.copy_(before_k); c.v.copy_(before_v)
                step()
                torch.cuda.synchronize()
                assert torch.equal(torch.nan_to_num(c.k.float()), torch.nan_to_num(cache[0].float()))
                assert all(torch.equal(s[n], t) for n, t in got.items())
            lens = lens + got["k"].cpu().numpy() + 1
    assert len(set(accepted)) > 1
