"""The paged 8-bit cache (cache_plan, cache_write, cache_decode) against its definitions in
numpy, 64 bits (tests/cache_ref.py).  Plans, codes, scales and key sums have to be equal;
decode is within the bound that cache_ref.check_decode counts."""
import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2502_13189_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def to_gpu(pool):
    f8 = torch.float8_e4m3fn
    t = lambda x: torch.from_numpy(x.copy()).to(DEV)  # noqa: E731
    return binding.PagedCache(t(pool.k).view(f8), t(pool.v).view(f8), t(pool.k_scale),
                              t(pool.v_scale), t(pool.k_sum))


def to_host(cache, pool):
    got = pool.copy()
    got.k, got.v = (x.view(torch.uint8).cpu().numpy() for x in (cache.k, cache.v))
    got.k_scale, got.v_scale, got.k_sum = (x.cpu().numpy() for x in cache[2:])
    return got


def same_pools(got, want):
    for name in ("k", "v"):
        a, b = getattr(got, name), getattr(want, name)
        # (the sign of a zero that a rounding leaves is not part of the definition)
        bad = (a != b) & ~((a & 127 == 0) & (b & 127 == 0)) & ~((a & 127 == 127) & (b & 127 == 127))
        assert not bad.any(), (name, np.argwhere(bad)[:4], a[bad][:4], b[bad][:4])
    for name in ("k_scale", "v_scale", "k_sum"):
        np.testing.assert_array_equal(getattr(got, name), getattr(want, name), err_msg=name)


# -------------------------------------------------------------------- plan
def check_plan(add, lens, table, free, num_free, page, T, in_place=False, wide=0):
    g_add, g_lens, g_nf = i32(add), i32(lens), i32([num_free])
    if wide:  # rows of a wider tensor
        big = i32(np.full((table.shape[0], table.shape[1] + wide), -7))
        g_table = big[:, :table.shape[1]]
        g_table.copy_(i32(table))
    else:
        g_table = i32(table)
    g_free = i32(free)
    more = dict(lens_out=g_lens, num_free_out=g_nf) if in_place else {}
    p = binding.cache_plan(g_add, g_lens, g_table, g_free, g_nf, page, T, **more)
    w_table, w_free = np.array(table), np.array(free)
    cu, slots, new, n, refused = ref.plan(add, lens, w_table, w_free, num_free, page, T)
    np.testing.assert_array_equal(p.cu_new.cpu(), cu)
    np.testing.assert_array_equal(p.slots.cpu(), slots)
    np.testing.assert_array_equal(p.lens.cpu(), new)
    assert int(p.num_free) == n and int(p.refused) == refused
    np.testing.assert_array_equal(g_table.cpu(), w_table)
    np.testing.assert_array_equal(g_free.cpu(), w_free)
    if wide:
        assert bool((big[:, table.shape[1]:] == -7).all())
    if in_place:
        assert p.lens is g_lens and p.num_free is g_nf
    else:
        np.testing.assert_array_equal(g_lens.cpu(), lens)


def some_batch(rng, S, W, page, spare):
    """Random requests with their pages, and the free list."""
    lens = rng.integers(0, W * page + 1, S)
    lens[rng.random(S) < 0.2] = 0
    held = -(-lens // page)
    N = int(held.sum()) + spare
    ids = rng.permutation(N)
    table = rng.integers(-5, N + 5, (S, W))  # entries past a request's pages hold anything
    at = 0
    for s in range(S):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
    free = np.concatenate([ids[at:], rng.integers(0, N, at)])
    return lens, table, free, N - at


@pytest.mark.parametrize("S,W,page,spare,most,slack", [
    (1, 1, 64, 1, 1, 0), (3, 4, 64, 5, 70, 2), (17, 6, 128, 0, 3, 0), (64, 9, 192, 20, 200, 5),
    (65, 3, 64, 200, 2, 1), (300, 5, 256, 100, 400, -50), (1500, 2, 64, 300, 40, 7),
    (4096, 3, 64, 500, 9, 0), (4096, 3, 64, 700, 90, 0), (4000, 9, 64, 2000, 300, 0), (9, 400, 64, 4000, 9000, 100), (2, 3000, 64, 6000, 150000, -1),
    (4096, 3, 64, 600, 4, 3), (3000, 2, 64, 100, 1, -5), (70, 5, 192, 9, 4, 9000),
    (3000, 60, 64, 9000, 1000, 30),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(S, W, page, spare, most, slack, in_place):
    for seed in range(3):
        rng = np.random.default_rng(seed + 10 * S + W)
        lens, table, free, n = some_batch(rng, S, W, page, spare)
        add = rng.integers(0, most + 1, S)
        add[rng.random(S) < 0.25] = 0
        add[rng.random(S) < 0.15] = -1 - seed
        T = max(0, int(np.maximum(add, 0).sum()) + slack)
        check_plan(add, lens, table, free, n, page, T, in_place, wide=seed * 3)


@pytest.mark.parametrize("S,W,page,spare,most,slack", [
    (256, 40, 64, 3000, 600, 11), (257, 40, 64, 3000, 600, 0), (200, 9, 192, 100, 200, -300),
    (256, 70, 128, 9000, 4, 70000), (100, 300, 64, 8000, 9000, 5), (1, 2000, 64, 2000, 100000, 1),
    (30, 200, 256, 500, 20000, 700), (200, 80, 192, 1000, 900, -5000), (9, 90, 64, 300, 5000, 60000),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_of_long_steps(S, W, page, spare, most, slack, in_place):
    """Steps of more tokens than one work-group writes; requests that end and are refused among
    them, and such as begin on a page's last token."""
    for seed in range(2):
        rng = np.random.default_rng(seed + 10 * S + W)
        lens, table, free, n = some_batch(rng, S, W // 2, page, spare)
        table = np.concatenate([table, rng.integers(-5, n, (S, W - W // 2))], 1)
        lens[lens % page == 1] -= 1
        add = rng.integers(most // 2, most + 1, S)
        add[rng.random(S) < 0.1] = 0
        add[rng.random(S) < 0.2] = -1
        add[0] = most
        T = int(np.maximum(add, 0).sum()) + slack
        assert T > 8192
        check_plan(add, lens, table, free, n, page, T, in_place, wide=seed)


def test_plan_of_nothing():
    check_plan([], [], np.zeros((0, 3), int), np.arange(5), 4, 64, 3)
    check_plan([0, 0], [5, 0], np.zeros((2, 3), int), np.arange(5), 4, 64, 0)
    check_plan([1, 1], [63, 64], np.array([[4, 0], [3, 0]]), np.zeros(0, int), 0, 64, 2)


def test_plan_of_nothing_in_long_steps():
    """No requests, none that gets a token, and none that is granted one, with slots for many."""
    for T in (9000, 70000):
        check_plan([], [], np.zeros((0, 3), int), np.arange(5), 4, 64, T)
        check_plan([0, -1, 0], [5, 64, 0], np.array([[1, 9], [3, 9], [9, 9]]), np.arange(5), 3, 64, T)
        check_plan([200, 20000], [5, 0], np.array([[1, 9], [9, 9]]), np.arange(5), 3, 64, T)


def test_plan_returns_then_takes():
    """The pages of a request that ends are what the next one gets; a request that asks for
    too much on its own does not starve the ones after it, one that finds the list short
    does (those that need a page)."""
    table = np.array([[7, 8, 9], [5, 0, 0], [6, 0, 0], [2, 0, 0]])
    check_plan([-1, 65, 1, 100], [130, 64, 10, 64], table, np.array([1, 3, 4] + [0] * 7), 1, 64, 200)
    check_plan([0, 500, 1, 1], [130, 64, 64, 64], table, np.array([1, 3, 4] + [0] * 7), 2, 64, 600)
    check_plan([0, 100, 1, 1], [130, 64, 64, 10], table, np.array([1] + [0] * 9), 1, 64, 600)


def test_plan_bounds_bad_state():
    """Lengths and counts outside their ranges are cut to them: nothing outside the tensors is
    touched."""
    guard = i32(np.full(64, 77))
    lens, table, free = guard[8:11], guard[16:22].view(3, 2), guard[32:36]
    lens.copy_(i32([-5, 10 ** 9, 3]))
    table.copy_(i32([[0, 1], [2, 3], [1, 0]]))
    free.copy_(i32([0, 1, 2, 3]))
    p = binding.cache_plan(i32([1, -1, 2 ** 31 - 1]), lens, table, free, i32([99]), 64, 4)
    torch.cuda.synchronize()
    assert p.lens.tolist() == [1, 0, 3] and int(p.refused) == 1
    assert p.cu_new.tolist() == [0, 1, 1, 4] and p.slots.tolist()[1:] == [-1, -1, -1]
    rest = torch.ones(64, dtype=torch.bool)
    rest[8:11] = rest[16:22] = rest[32:36] = False
    assert bool((guard.cpu()[rest] == 77).all())
    p = binding.cache_plan(i32([1, 0, 0]), lens, table, free, i32([-3]), 64, 4)
    assert int(p.num_free) == 0 and int(p.refused) == 1


# ------------------------------------------------------------------- write
def some_rows(rng, T, hkv, dtype, hard=True):
    x = rng.standard_normal((T, hkv, ref.D)) * np.exp(rng.standard_normal((T, hkv, 1)))
    if hard and T > 2:
        x[rng.random((T, hkv)) < 0.1] = 0.0
        x[rng.random(x.shape) < 0.002] *= 300.0
        x[rng.random(x.shape) < 0.01] *= 1e-4
    t = torch.from_numpy(x).to(DEV, dtype)
    return t, t.double().cpu().numpy()


def check_write(pool, slots, dtype, seed, hard=True, edit=None, strided=False):
    rng = np.random.default_rng(seed)
    T = len(slots)
    (k, nk), (v, nv) = (some_rows(rng, T, pool.hkv, dtype, hard) for _ in range(2))
    if edit is not None:
        edit(k, v)
        nk, nv = k.double().cpu().numpy(), v.double().cpu().numpy()
    if strided:  # heads of one fused projection
        qkv = torch.zeros((T, 2 * pool.hkv + 3, ref.D), dtype=dtype, device=DEV)
        qkv[:, 1:1 + pool.hkv], qkv[:, -pool.hkv:] = k, v
        k, v = qkv[:, 1:1 + pool.hkv], qkv[:, -pool.hkv:]
    cache = to_gpu(pool)
    g_slots = torch.tensor(np.asarray(slots), dtype=torch.int64, device=DEV)
    binding.cache_write(k, v, g_slots, cache)
    ref.write(nk, nv, slots, pool)
    same_pools(to_host(cache, pool), pool)
    binding.cache_write(k, v, g_slots, cache)  # again: nothing changes
    same_pools(to_host(cache, pool), pool)


def runs(pool, rng, spans):
    """Slots of runs (offset, tokens) on pages of their own, in no order, with rows that are
    left out between them."""
    pages = rng.permutation(pool.n)
    slots = []
    for (o, n), p in zip(spans, pages):
        slots += [int(p) * pool.page + o + i for i in range(n)]
        if rng.random() < 0.3:
            slots += [-1] * int(rng.integers(1, 4))
    return slots


def filled(pool, seed):
    """The pool with every page written."""
    rng = np.random.default_rng(seed)
    n = pool.n * pool.page
    ref.write(rng.standard_normal((n, pool.hkv, ref.D)), rng.standard_normal((n, pool.hkv, ref.D)) * 3,
              np.arange(n), pool)
    return pool


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [64, 128, 192, 256])
def test_write_runs(page, dtype):
    rng = np.random.default_rng(page)
    pool = filled(ref.Pool(12, 2, page), 1)
    spans = [(0, page), (0, 1), (1, 1), (page - 1, 1), (0, page - 1), (3, page - 3), (17, 30),
             (page // 2, page // 2), (page - 5, 3), (31, 33), (0, 32), (32, 5)]
    check_write(pool, runs(pool, rng, spans), dtype, page + 1)


@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_write_prompts_fresh(hkv):
    """Whole prompts into pages that were never written (NaN everywhere)."""
    rng = np.random.default_rng(hkv)
    for page, tokens in ((64, 300), (192, 500), (128, 1)):
        pool = ref.Pool(10, hkv, page)
        pages = rng.permutation(10)
        slots = [int(pages[t // page]) * page + t % page for t in range(tokens)]
        check_write(pool, slots, torch.bfloat16, tokens + hkv)


def test_write_token_by_token():
    """A page filled one token at a time, with rising and falling sizes: older tokens are
    rescaled where the scale grows, and only then."""
    pool = ref.Pool(3, 2, 64)
    rng = np.random.default_rng(5)
    cache = to_gpu(pool)
    for t in range(70):
        page, o = (2, t) if t < 64 else (0, t - 64)
        x = rng.standard_normal((1, 2, ref.D)) * 2.0 ** rng.integers(-12, 12)
        k = torch.from_numpy(x).to(DEV, torch.bfloat16)
        v = torch.from_numpy(x[..., ::-1] * 7).to(DEV, torch.bfloat16)
        slot = [page * 64 + o]
        binding.cache_write(k, v, torch.tensor(slot, device=DEV), cache)
        ref.write(k.double().cpu().numpy(), v.double().cpu().numpy(), slot, pool)
        same_pools(to_host(cache, pool), pool)


@pytest.mark.parametrize("page", [64, 128, 192, 256])
def test_write_single_tokens(page):
    """A decode step's tokens: one for each of many pages, at every kind of offset, with sizes
    that make older tokens keep their scale or lose it; older and new keys with NaN; runs of
    two and more, and rows that are left out, between them."""
    rng = np.random.default_rng(page)
    for spans, dtype in (([(int(o), 1) for o in rng.integers(0, page, 60)], torch.bfloat16),
                         ([(o, 1) for o in (0, 1, 7, 8, 31, 32, 33, 62, 63, page - 1)], torch.float32),
                         ([(int(o), int(min(n, page - o))) for o, n in zip(
                             rng.integers(0, page, 90), rng.choice([1, 1, 1, 2, 5, 64], 90))], torch.bfloat16)):
        pool = filled(ref.Pool(len(spans) + 2, 3, page), 5)
        pool.k[3, :, 2, 5] = pool.k[7, 1, page - 1, 9] = 0x7f
        slots = runs(pool, rng, spans)

        def edit(k, v):
            k *= torch.from_numpy(2.0 ** rng.integers(-8, 9, (len(k), 1, 1))).to(DEV, dtype)
            k[1, 0, 3], v[2, 2, 100], v[4] = float("nan"), float("inf"), 0.0
        check_write(pool, slots, dtype, page + 2, edit=edit)


def test_write_extremes():
    """Zeros, subnormals, the type's largest values, infinities and NaN."""
    def edit(k, v):
        k[0] = 0.0
        k[1, 0] = 1e-38
        k[2, :, ::3] = 3.3e38
        k[3, 1, 5] = float("inf")
        k[4, 0, 7] = float("nan")
        v[2, :, 0] = -float("inf")
        v[5] = 1e-30
        v[6, 0] = 448.0
        v[6, 1] = 449.0
    for spans in ([(0, 64)], [(0, 1)] * 8, [(5, 3), (0, 5), (60, 4)], [(1, 1)] * 7):
        pool = filled(ref.Pool(9, 2, 64), 3)
        check_write(pool, runs(pool, np.random.default_rng(1), spans)[:80], torch.bfloat16, 7,
                    edit=lambda k, v: edit(k, v) if len(k) > 6 else None)
    pool = filled(ref.Pool(2, 2, 64), 4)
    check_write(pool, list(range(40)), torch.float32, 8, edit=edit)


def test_write_ties():
    """Codes halfway between two: to the even one."""
    pool = ref.Pool(2, 1, 64)
    base = ref.F8[:126]
    mids = np.zeros((2, 1, ref.D))
    mids[0, 0, :126] = (base + ref.F8[1:127]) / 2
    mids[1, 0, :126] = -mids[0, 0, :126]
    mids[:, 0, 127] = 448.0
    k = torch.from_numpy(mids).to(DEV, torch.float32)
    cache = to_gpu(pool)
    slots = [0, 1]
    binding.cache_write(k, -k, torch.tensor(slots, device=DEV), cache)
    ref.write(mids, -mids, slots, pool)
    assert pool.k_scale[0, 0] == 1.0
    same_pools(to_host(cache, pool), pool)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_write_many_rows_in_no_order(dtype):
    """Many runs (windows of several tokens), fused inputs, slots outside the pool."""
    pool = filled(ref.Pool(700, 2, 64), 9)
    rng = np.random.default_rng(2)
    spans = [(0, 64)] * 120 + [(int(o), int(rng.integers(1, 65 - o))) for o in rng.integers(0, 64, 500)]
    order = rng.permutation(len(spans))
    slots = runs(pool, rng, [spans[i] for i in order])
    slots[0:0] = [700 * 64, 1 << 40, -(1 << 40)]  # (between runs: a page has one run per call)
    check_write(pool, slots, dtype, 11, strided=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [64, 128, 192, 256])
def test_write_windows_of_a_page(page, dtype):
    """Rows and heads enough that a work-group takes a page's rows: whole pages, prompts cut
    anywhere, single tokens.  A page's bits do not depend on what else a call writes, so they
    are those of calls of a few hundred rows each, which the tests above hold to the definition."""
    rng, hkv = np.random.default_rng(page), 16
    spans = [(0, page)] * (13000 // page) + [(int(o), int(rng.integers(1, page + 1 - o)))
                                             for o in rng.integers(0, page, 60)]
    spans += [(int(o), 1) for o in rng.integers(0, page, 300)]
    spans = [spans[i] for i in rng.permutation(len(spans))] + [(0, page)] * (4000 // page)
    spans += [(int(o), 1) for o in rng.integers(0, page, 300)]
    slots, cuts = [], [0]
    for (o, n), p in zip(spans, rng.permutation(len(spans) + 1)):
        slots += [int(p) * page + o + i for i in range(n)] + [-1] * int(rng.integers(0, 2))
        if len(slots) - cuts[-1] > 500:
            cuts.append(len(slots))
    assert len(slots) * hkv / 64 >= 4096
    gen = torch.Generator(device=DEV).manual_seed(page)
    one = binding.cache_new(len(spans) + 1, hkv, page, device=DEV)
    for x in one:  # (codes of any kind but NaN)
        x.copy_(torch.randn(x.shape, generator=gen, device=DEV).to(x.dtype))
    one.k_scale.copy_(2.0 ** torch.randint(-12, 1, one.k_scale.shape, generator=gen, device=DEV))
    one.v_scale.copy_(2.0 ** torch.randint(-12, 1, one.k_scale.shape, generator=gen, device=DEV))
    many = binding.PagedCache(*(x.clone() for x in one))
    k, v = (torch.randn((len(slots), hkv, 128), generator=gen, device=DEV).to(dtype) for _ in range(2))
    k[3, 10, 3], v[70, 15, 100], v[-2, 5, 5] = float("nan"), float("inf"), -float("inf")
    slots = torch.tensor(slots, device=DEV)
    binding.cache_write(k, v, slots, one)
    for lo, hi in zip(cuts, cuts[1:] + [len(slots)]):
        binding.cache_write(k[lo:hi], v[lo:hi], slots[lo:hi], many)
    for x, y in zip(one, many):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_write_into_a_layer_of_a_larger_pool():
    """Pages and heads with strides: the second of three layers, K and V side by side."""
    pool = filled(ref.Pool(6, 2, 128), 2)
    f8 = torch.float8_e4m3fn
    both = torch.full((6, 3, 2, 2, 128 * 128), 0x55, dtype=torch.uint8, device=DEV)
    kv = both[:, 1]
    kv[:, 0] = torch.from_numpy(pool.k).to(DEV).view(6, 2, -1)
    kv[:, 1] = torch.from_numpy(pool.v).to(DEV).view(6, 2, -1)
    c = to_gpu(pool)
    cache = binding.PagedCache(kv[:, 0].unflatten(2, (128, 128)).view(f8),
                               kv[:, 1].unflatten(2, (2, 128, 64)).view(f8), *c[2:])
    rng = np.random.default_rng(3)
    slots = runs(pool, rng, [(0, 128), (5, 60), (127, 1), (64, 64)])
    (k, nk), (v, nv) = (some_rows(rng, len(slots), 2, torch.bfloat16) for _ in range(2))
    binding.cache_write(k, v, torch.tensor(slots, device=DEV), cache)
    ref.write(nk, nv, slots, pool)
    same_pools(to_host(cache, pool), pool)
    assert bool((both[:, 0] == 0x55).all()) and bool((both[:, 2] == 0x55).all())
    q = torch.randn((2, 4, 128), device=DEV).to(torch.bfloat16)
    table, lens = np.array([[1, 2, 0], [4, 0, 0]]), [300, 128]
    out, lse = binding.cache_decode(q, cache, i32(table), i32(lens), 128, 2)
    want = ref.decode(q.double().cpu().numpy(), pool, table, lens, 128, 2)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)


# ------------------------------------------------------------------ decode
def some_cache(rng, lens, hkv, page, W, spread=1.0):
    """A pool that holds requests of these lengths (everything else is NaN), and their
    table (entries past a request's pages hold anything)."""
    held = [-(-max(x, 0) // page) for x in lens]
    n = sum(held) + 3
    pool = ref.Pool(n, hkv, page)
    ids = rng.permutation(n)
    table = rng.integers(-(2 ** 31), 2 ** 31, (len(lens), W))
    at = 0
    for s, L in enumerate(lens):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
        if L <= 0:
            continue
        # the keys of 64 tokens share an offset, so that blocks differ
        k = rng.standard_normal((L, hkv, ref.D)) + spread * rng.standard_normal((-(-L // 64), hkv, ref.D)).repeat(64, 0)[:L]
        v = rng.standard_normal((L, hkv, ref.D)) * np.exp(rng.standard_normal((L, 1, 1)))
        t = np.arange(L)
        ref.write(k, v, table[s][t // page] * page + t % page, pool)
    return pool, table


def check(pool, table, lens, hq, block, topk, rng, what="", **more):
    q = torch.from_numpy(rng.standard_normal((len(lens), hq, ref.D))).to(DEV, torch.bfloat16)
    cache = to_gpu(pool)
    out, lse = binding.cache_decode(q, cache, i32(table), i32(lens), block, topk, **more)
    want = ref.decode(q.double().cpu().numpy(), pool, table, lens, block, topk)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want, what)
    return q, cache, out, lse


LENS = [1, 63, 64, 65, 0, 127, 128, 129, 700, -4, 333, 2, 17]


# A short table row is one work-group's, a long one is split over the chip: most tests run
# with their requests in tables of both kinds.
WIDTHS = [13, 400]


@pytest.mark.parametrize("W", WIDTHS)
@pytest.mark.parametrize("page", [64, 128, 192, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (8, 2), (16, 1), (10, 2)])
def test_decode_full(page, hq, hkv, W):
    rng = np.random.default_rng(page + hq)
    pool, table = some_cache(rng, LENS, hkv, page, W)
    check(pool, table, LENS, hq, 0, 0, rng)


@pytest.mark.parametrize("page,block,topk", [(64, 64, 3), (64, 128, 2), (64, 64, 1), (128, 128, 4),
                                             (64, 192, 3), (192, 192, 2), (256, 256, 2),
                                             (64, 64, 9), (64, 64, 500)])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (16, 1)])
@pytest.mark.parametrize("W", WIDTHS)
def test_decode_moba(page, block, topk, hq, hkv, W):
    rng = np.random.default_rng(page + block + topk + hq)
    pool, table = some_cache(rng, LENS, hkv, page, W)
    check(pool, table, LENS, hq, block, topk, rng)


@pytest.mark.parametrize("lens,hq,hkv,page,block,topk", [
    ([9000], 4, 1, 64, 0, 0),            # one request over every share
    ([9000, 1, 40, 5000], 2, 2, 128, 0, 0),
    ([9000], 4, 1, 64, 256, 5),
    ([200] * 70, 2, 1, 64, 0, 0),        # shares that hold several requests
    ([200] * 70, 2, 1, 64, 64, 2),
    ([18000], 2, 1, 64, 64, 7),          # 282 blocks: more than the first selection holds
    ([70000, 130], 1, 1, 64, 64, 30),    # 1094 blocks
    ([300] * 150 + [8000], 4, 4, 64, 512, 3),  # many rows: a work-group each, one of them long
    ([64 * 126, 5, 7000], 16, 1, 64, 64, 5),   # the most blocks a work-group gates
    ([1000, 77, 2048] * 20, 6, 2, 128, 0, 0),
    ([150, 3, 700] * 60, 4, 4, 64, 0, 0),
])
def test_decode_splits(lens, hq, hkv, page, block, topk):
    rng = np.random.default_rng(len(lens) + hq)
    W = -(-max(lens) // page) + 2
    pool, table = some_cache(rng, lens, hkv, page, W)
    check(pool, table, lens, hq, block, topk, rng)


@pytest.mark.parametrize("lens,hq,hkv,page,block,topk", [
    ([300, 64, 1] * 50 + [9000], 4, 4, 64, 64, 3),   # a work-group for each of 604 rows, unjoined
    ([300, 0, 5000, -1] * 20, 12, 4, 64, 64, 9),     # two work-groups a row, some of them idle
    ([12345, 3, 0, 7000], 16, 1, 128, 1024, 6),      # many, of long blocks
    ([20000, 19999], 4, 1, 64, 2048, 1),             # the current block alone: no gate
    ([16500], 3, 1, 64, 64, 257),                    # all past blocks but one
])
def test_decode_parts(lens, hq, hkv, page, block, topk):
    rng = np.random.default_rng(len(lens) + topk)
    W = max(-(-max(lens) // page) + 2, 131)
    pool, table = some_cache(rng, lens, hkv, page, W)
    check(pool, table, lens, hq, block, topk, rng)


@pytest.mark.parametrize("lens", [[300, 0, 1, 900, 64] * 13, [100] * 64, [300, 0, 1, 900] * 16,
                                  [0] * 70 + [2000], [0] * 63 + [2000]])
def test_decode_more_requests_than_shares(lens):
    """32 kv-heads have 64 shares each, for up to 64 requests and for more."""
    rng = np.random.default_rng(len(lens))
    pool, table = some_cache(rng, lens, 32, 64, 80)
    check(pool, table, lens, 32, 0, 0, rng)


@pytest.mark.parametrize("W", [257, 1025, 2049, 4096])
@pytest.mark.parametrize("topk", [1, 2, 33, 65, 66, 70])
def test_decode_selection(topk, W):
    """Wide tables, few and many blocks chosen, pages with equal sums and with NaN among them,
    sums that differ in their last bits alone or by many powers of two."""
    rng = np.random.default_rng(topk)
    lens = [5000, 63, 4200, 4200]
    pool, table = some_cache(rng, lens, 2, 64, W)
    for j in range(3, 30):  # (equal scores, as another page's)
        pool.k_sum[table[0, j]] = pool.k_sum[table[0, 2]]
    pool.k_sum[table[0, 40]] = np.nan
    for j in range(60):
        pool.k_sum[table[2, j]] = pool.k_sum[table[2, 0]] * np.float32(1 + (j * 7 % 60) * 2.0 ** -22)
        pool.k_sum[table[3, j]] *= np.float32(2.0 ** ((j * 13) % 60 - 30))
    check(pool, table, lens, 4, 64, topk, rng)


@pytest.mark.parametrize("lens", [[2049], [2112, 1], [4096], [4097], [1000, 0, 1100], [64] * 33, [64] * 32])
def test_decode_share_of_two_steps(lens):
    """32 kv-heads have 64 shares each: up to 32 steps, up to 64 and more."""
    rng = np.random.default_rng(sum(lens))
    pool, table = some_cache(rng, lens, 32, 64, 80)
    check(pool, table, lens, 64, 0, 0, rng)


@pytest.mark.parametrize("W", WIDTHS)
@pytest.mark.parametrize("topk", [0, 2, 3])
def test_decode_bad_table_entries(topk, W):
    """Entries that are no page are left out; a request all of whose pages are attends nothing."""
    rng = np.random.default_rng(4)
    lens = [300, 64, 500, 130]
    pool, table = some_cache(rng, lens, 2, 64, W)
    for s, j, x in ((0, 1, -1), (0, 4, pool.n), (1, 0, 2 ** 31 - 1), (2, 0, -2 ** 31), (2, 7, -1)):
        table[s, j] = x
    check(pool, table, lens, 4, 128, topk, rng)


def test_decode_lengths_past_the_table():
    rng = np.random.default_rng(6)
    pool, table = some_cache(rng, [192, 128], 1, 64, 3)
    table[1, 2] = -1
    check(pool, table, [10 ** 9, 128], 2, 0, 0, rng)
    check(pool, table, [2 ** 31 - 1, 128], 2, 64, 2, rng)


@pytest.mark.parametrize("W", WIDTHS)
def test_decode_equal_scores_take_the_lower_block(W):
    """Every block holds the same keys, so all scores are equal; values tell the blocks apart."""
    rng = np.random.default_rng(8)
    pool, table = some_cache(rng, [700], 1, 64, W)
    for j in range(10):
        pool.k[table[0, j]] = pool.k[table[0, 0]]
        pool.k_scale[table[0, j]] = pool.k_scale[table[0, 0]]
        pool.k_sum[table[0, j]] = pool.k_sum[table[0, 0]]
    for topk in (2, 4, 10):
        check(pool, table, [700], 4, 64, topk, rng, "top-%d" % topk)


@pytest.mark.parametrize("W", WIDTHS)
def test_decode_scores_that_are_no_numbers(W):
    """A block whose key sum is NaN counts as the lowest."""
    rng = np.random.default_rng(9)
    pool, table = some_cache(rng, [700], 1, 64, W)
    pool.k_sum[table[0, 3]] = np.nan
    pool.k_sum[table[0, 5], 0, 0] = np.inf
    q, cache, out, _ = check(pool, table, [700], 2, 64, 4, rng)
    assert bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("W", WIDTHS)
def test_decode_scales_far_apart(W):
    """Pages whose scales differ by 2^40, and very large logits."""
    rng = np.random.default_rng(10)
    pool, table = some_cache(rng, [500, 100], 2, 64, W)
    pool.v_scale[table[0, 2]] *= 2.0 ** 40
    pool.v_scale[table[0, 3]] *= 2.0 ** -40
    pool.k_scale[table[0, 4]] *= 2.0 ** 4
    pool.k_scale[table[1, 1]] *= 2.0 ** -30
    pool.k_scale[table[0, 5]] *= 1.3  # (any scale is read, not only powers of two)
    check(pool, table, [500, 100], 4, 0, 0, rng)


@pytest.mark.parametrize("W", [32, 400])
def test_decode_one_key_far_above(W):
    """A late key far above all others: the running maximum moves."""
    rng = np.random.default_rng(11)
    pool, table = some_cache(rng, [2000], 1, 64, W)
    q = rng.standard_normal((1, 4, ref.D))
    for at, size in ((100, 2.0), (900, 4.0), (1999, 6.0)):
        k = (q[0, at % 4] * size)[None, None]
        ref.write(k, rng.standard_normal(k.shape), [int(table[0, at // 64]) * 64 + at % 64], pool)
    g_q = torch.from_numpy(q).to(DEV, torch.bfloat16)
    out, lse = binding.cache_decode(g_q, to_gpu(pool), i32(table), i32([2000]), 0, 0)
    want = ref.decode(g_q.double().cpu().numpy(), pool, table, [2000], 0, 0)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)


@pytest.mark.parametrize("W", WIDTHS)
@pytest.mark.parametrize("topk", [0, 3])
def test_decode_layouts(topk, W):
    """Strided q, out in q's own memory, rows of a wider table, a used workspace, twice."""
    rng = np.random.default_rng(12)
    lens = [300, 0, 129, 700]
    pool, table = some_cache(rng, lens, 2, 64, W)
    cache = to_gpu(pool)
    big = torch.randn((4, 12, 128), device=DEV).to(torch.bfloat16)
    q = big[:, 2:10]
    keep = big.clone()
    wide = i32(np.full((4, W + 8), 2 ** 30))
    wide[:, 3:3 + W] = i32(table)
    n = binding.cache_decode_workspace_bytes(4, W, 8, 2, 64, 64, topk)
    ws = torch.full((n + 64,), 0xff, dtype=torch.uint8, device=DEV)
    lse = torch.empty((8, 4), device=DEV)
    want = ref.decode(q.double().cpu().numpy(), pool, table, lens, 64, topk)
    a, la = binding.cache_decode(q, cache, wide[:, 3:3 + W], i32(lens), 64, topk)
    binding.cache_decode(q, cache, wide[:, 3:3 + W], i32(lens), 64, topk, out=q, lse=lse, workspace=ws[:n])
    torch.cuda.synchronize()
    assert torch.equal(a, q) and torch.equal(la, lse)
    ref.check_decode(q.double().cpu().numpy(), lse.double().cpu().numpy(), want)
    assert torch.equal(big[:, :2], keep[:, :2]) and torch.equal(big[:, 10:], keep[:, 10:])
    assert bool((ws[n:] == 0xff).all())


def test_decode_offsets_past_32_bits():
    """Pages far into a pool of more than 4 GiB: K at offsets above 2^32 bytes."""
    rng = np.random.default_rng(13)
    lens = [300, 90]
    small, table = some_cache(rng, lens, 1, 64, 5)
    far = 600_000
    cache = binding.cache_new(far + small.n, 1, 64, device=DEV)
    c = to_gpu(small)
    for big, s in zip(cache, c):
        big.view(torch.uint8)[far:].copy_(s.view(torch.uint8))
    q = torch.randn((2, 4, 128), device=DEV).to(torch.bfloat16)
    want = ref.decode(q.double().cpu().numpy(), small, table, lens, 64, 2)
    t = i32(np.where((table >= 0) & (table < small.n), table + far, -1))
    out, lse = binding.cache_decode(q, cache, t, i32(lens), 64, 2)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)
    k = torch.randn((2, 1, 128), device=DEV).to(torch.bfloat16)
    slots = np.array([int(table[0, 4]) * 64 + 44, int(table[1, 1]) * 64 + 26])
    binding.cache_write(k, k, torch.tensor(slots + far * 64, device=DEV), cache)
    nk = k.double().cpu().numpy()
    ref.write(nk, nk, slots, small)
    got = binding.PagedCache(*(x.view(torch.uint8)[far:].clone().view(x.dtype) for x in cache))
    same_pools(to_host(got, small), small)


# ---------------------------------------------------------------- together
def test_agrees_with_decode_over_a_packed_cache():
    """Keys and values that e4m3 holds exactly: cache_decode over the pages and decode over the
    packed bf16 cache are the same function (each within its rounding to bf16)."""
    rng = np.random.default_rng(14)
    lens, hq, hkv = [1000, 300, 64, 1], 8, 2
    T = sum(lens)
    k = torch.from_numpy(rng.integers(-8, 9, (T, hkv, 128)) / 8.0).to(DEV, torch.bfloat16)
    v = torch.from_numpy(rng.integers(-8, 9, (T, hkv, 128)) / 4.0).to(DEV, torch.bfloat16)
    q = torch.randn((4, hq, 128), device=DEV).to(torch.bfloat16)
    cache = binding.cache_new(40, hkv, 64, device=DEV)
    table = torch.zeros((4, 20), dtype=torch.int32, device=DEV)
    free = i32(rng.permutation(40))
    p = binding.cache_plan(i32(lens), i32([0] * 4), table, free, i32([40]), 64, T)
    binding.cache_write(k, v, p.slots, cache)
    cu = p.cu_new.cpu()
    for topk in (0, 3):
        a, la = binding.cache_decode(q, cache, table, p.lens, 128, topk)
        b, lb = binding.decode(q, k, v, cu, 128, topk)
        a, b = a.double(), b.double()
        # two roundings to bf16 (2^-8 each) and decode's weights in one bf16 term
        tol = 2.0 ** -7 * b.abs() + 2.0 ** -8 * v.double().abs().max()
        assert bool(((a - b).abs() <= tol).all())
        assert float((la - lb).abs().max()) <= 1e-4


@pytest.mark.parametrize("W", [5, 200])
def test_serving_steps_captured(W):
    """Plan, write and decode as one captured step, replayed while requests grow, end, enter
    and are refused; eager work and synchronizations between the replays.  Each replay is
    compared with the definitions."""
    rng = np.random.default_rng(15)
    S, hq, hkv, page, N, T = 6, 8, 2, 64, 14, 160
    pool = ref.Pool(N, hkv, page)
    cache = to_gpu(pool)
    w_table, w_free, w_lens, n = np.full((S, W), -1), rng.permutation(N), np.zeros(S, int), N
    table, free, lens, nf = i32(w_table), i32(w_free), i32(w_lens), i32([n])
    add = i32([0] * S)
    k, v = (torch.zeros((T, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.zeros((S, hq, 128), dtype=torch.bfloat16, device=DEV)

    def step():
        p = binding.cache_plan(add, lens, table, free, nf, page, T, lens_out=lens, num_free_out=nf)
        binding.cache_write(k, v, p.slots, cache)
        return [p, binding.cache_decode(q, cache, table, lens, 0, 0),
                binding.cache_decode(q, cache, table, lens, 64, 2)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()  # (adds nothing)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    steps = [[130, 20, 0, 0, 0, 0], [1, 1, 5, 0, 100, 0], [1] * 6, [1, -1, 1, 1, 1, 1], [0, 0, 0, 90, 0, 30],
             [-1, 64, 1, 1, 1, 1], [1, 0, 0, 0, 64, 0], [-1, -1, -1, -1, -1, 120], [0, 150, 0, 0, 9, 0],
             [1, 1, 1, 1, 1, 1]]
    for i, a in enumerate(steps):
        add.copy_(i32(a))
        for x in (k, v, q):
            x.copy_(torch.from_numpy(rng.standard_normal(x.shape)).to(DEV))
        torch.randn(1000, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        cu, slots, w_lens, n, refused = ref.plan(a, w_lens, w_table, w_free, n, page, T)
        ref.write(k.double().cpu().numpy(), v.double().cpu().numpy(), slots, pool)
        p = got[0]
        np.testing.assert_array_equal(p.slots.cpu(), slots)
        np.testing.assert_array_equal(lens.cpu(), w_lens)
        np.testing.assert_array_equal(table.cpu(), w_table)
        np.testing.assert_array_equal(free.cpu(), w_free)
        assert int(nf) == n and int(p.refused) == refused
        same_pools(to_host(cache, pool), pool)
        for (out, lse), (b, topk) in zip(got[1:], ((0, 0), (64, 2))):
            want = ref.decode(q.double().cpu().numpy(), pool, w_table, w_lens, b, topk)
            ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want, "step %d" % i)


def test_decode_on_two_streams():
    """Calls on streams of their own, workspaces by default: the same results, bit for bit."""
    rng = np.random.default_rng(16)
    lens = [5000, 100, 2000]
    pool, table = some_cache(rng, lens, 2, 64, 80)
    cache, t, ln = to_gpu(pool), i32(table), i32(lens)
    qs = [torch.randn((3, 8, 128), device=DEV).to(torch.bfloat16) for _ in range(2)]
    want = [binding.cache_decode(q, cache, t, ln, 64, topk) for q, topk in zip(qs, (0, 3))]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for q, topk, st in zip(qs, (0, 3), streams):
            got.append(binding.cache_decode(q, cache, t, ln, 64, topk, stream=st))
    torch.cuda.synchronize()
    for i, (o, l) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(l, want[i % 2][1])


def test_two_graphs_share_a_workspace():
    """Two captured decodes of different shapes with one workspace between them, replayed in
    turn (one stream): each finds nothing of the other's."""
    rng = np.random.default_rng(17)
    batches = []
    for lens, hq, hkv, topk in (([9000, 70, 300], 4, 1, 0), ([5000, 6100], 8, 2, 3)):
        pool, table = some_cache(rng, lens, hkv, 64, 300)
        q = torch.randn((len(lens), hq, 128), device=DEV).to(torch.bfloat16)
        n = binding.cache_decode_workspace_bytes(len(lens), 300, hq, hkv, 64, 64, topk)
        batches.append([q, to_gpu(pool), i32(table), i32(lens), 64, topk, n])
    ws = torch.full((max(b[-1] for b in batches),), 0xff, dtype=torch.uint8, device=DEV)
    want = [binding.cache_decode(*b[:-1]) for b in batches]
    torch.cuda.synchronize()
    graphs = []
    for b in batches:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = binding.cache_decode(*b[:-1], workspace=ws)
        graphs.append((g, got))
    for i in (0, 1, 1, 0, 1, 0, 0):
        g, got = graphs[i]
        got[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[i][0]) and torch.equal(got[1], want[i][1])


def test_steps_on_a_stream_of_their_own():
    """Every call on a side stream passed in, outputs passed in and left out."""
    rng = np.random.default_rng(18)
    lens = [100, 64, 0, 17]
    T = sum(lens) + 5
    st = torch.cuda.Stream()
    k, v = (torch.randn((T, 2, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((4, 4, 128), device=DEV).to(torch.bfloat16)
    cache = binding.cache_new(9, 2, 64, device=DEV)
    table, free = i32(np.full((4, 3), -1)), i32(rng.permutation(9))
    add, zero, nf = i32(lens), i32([0] * 4), i32([9])
    slots = torch.empty((T,), dtype=torch.int64, device=DEV)
    torch.cuda.synchronize()
    p = binding.cache_plan(add, zero, table, free, nf, 64, T, slots=slots, stream=st)
    binding.cache_write(k, v, p.slots, cache, stream=st.cuda_stream)
    out, lse = binding.cache_decode(q, cache, table, p.lens, 64, 2, stream=st)
    st.synchronize()
    assert p.slots is slots
    pool = ref.Pool(9, 2, 64)
    w_table, w_free = np.full((4, 3), -1), free.cpu().numpy().copy()
    w_slots = ref.plan(lens, [0] * 4, w_table, w_free, 9, 64, T)[1]
    np.testing.assert_array_equal(slots.cpu(), w_slots)
    ref.write(k.double().cpu().numpy(), v.double().cpu().numpy(), w_slots, pool)
    want = ref.decode(q.double().cpu().numpy(), pool, w_table, lens, 64, 2)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)


def test_refusals_leave_everything():
    """What the library or the binding refuses touches nothing."""
    rng = np.random.default_rng(19)
    pool, table = some_cache(rng, [100, 30], 2, 64, 4)
    cache, t, ln = to_gpu(pool), i32(table), i32([100, 30])
    q = torch.randn((2, 4, 128), device=DEV).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)

    def refused(name, f, *args, **kw):
        with pytest.raises(binding.MobaError) as e:
            f(*args, **kw)
        assert e.value.name == name

    refused("MOBA_ERR_DTYPE", binding.cache_decode, q.float(), cache, t, ln, 64, 0)
    refused("MOBA_ERR_BLOCK_SIZE", binding.cache_decode, q, cache, t, ln, 96, 2, out=out)
    refused("MOBA_ERR_TOPK", binding.cache_decode, q, cache, t, ln, 64, -1, out=out)
    refused("MOBA_ERR_SHAPE", binding.cache_decode, q, cache, t[:1], ln, 64, 2, out=out)
    refused("MOBA_ERR_NO_MEMORY", binding.cache_decode, q, cache, t, ln, 64, 2, out=out,
            workspace=torch.empty((15,), dtype=torch.uint8, device=DEV))
    refused("MOBA_ERR_LAYOUT", binding.cache_decode, q, cache, t, ln, 64, 2,
            out=q.new_empty((2, 4, 256))[..., ::2])
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=DEV)
    slots = torch.tensor([0, 1, 2], device=DEV)
    refused("MOBA_ERR_DTYPE", binding.cache_write, x, x.float(), slots, cache)
    refused("MOBA_ERR_DTYPE", binding.cache_write, x, x, slots.int(), cache)
    refused("MOBA_ERR_SHAPE", binding.cache_write, x[:, :1], x[:, :1], slots, cache)
    refused("MOBA_ERR_UNSUPPORTED", binding.cache_plan, ln, ln, t, ln, ln[:1], 96, 4)
    for f, args in ((binding.cache_decode, (q, cache, t.cpu(), ln, 64, 0)),
                    (binding.cache_write, (x, x.cpu(), slots, cache)),
                    (binding.cache_plan, (ln, ln, t, ln.cpu(), ln[:1], 64, 4))):
        with pytest.raises(ValueError):
            f(*args)
    with pytest.raises(TypeError):
        binding.cache_write(x.half(), x.half(), slots, cache)
    with pytest.raises(TypeError):
        binding.cache_decode(q, cache[:4], t, ln, 64, 0)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
    same_pools(to_host(cache, pool), pool)
