"""The paged 8-bit cache at the edges of what its calls allow: weights that cancel, NaN in what some
heads attend, lengths near 2^31, cut-backs, table entries that are no page, and profiling
of captured calls."""
import math

import numpy as np
import pytest
import torch

import cache_ref as ref
from paper_2502_13189_amd import binding
from test_gpu_cache import DEV, WIDTHS, i32, some_cache, to_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()


@pytest.mark.parametrize("W", WIDTHS)
@pytest.mark.parametrize("topk", [0, 2])
def test_decode_weights_in_full(topk, W):
    """Two keys whose weighted values all but cancel, out = (a - b p) / (1 + p) with b p near a: what
    a rounding of the weights to fewer than 24 bits leaves shows in the result.

    In units of u = 2^-24: the logit, at most 0.91 in the log2 domain, is a sum of two exact
    products (2 u), times the scale (2 u) and rounded (u), so p is off by 5 * 0.91 * ln 2 = 3.2 u, and by
    4 u from its exponential; the bf16 terms of a weight make it up to u; six MFMAs add, each
    off by 2 u of the sum so far at most, which is at most a.  Of b p ~ a together less than 21 a u, that is less
    than 12 u of mass = (a + b p) / (1 + p).  The rounding to bf16 is 2^-8 of the result."""
    pairs = [(a, b) for a in range(8, 16) for b in range(a + 1, 16)]
    S = len(pairs)
    pool = ref.Pool(S, 1, 64)
    k, v, q = np.zeros((2 * S, 1, 128)), np.zeros((2 * S, 1, 128)), torch.zeros((S, 1, 128), dtype=torch.float64)
    slots = [s * 64 + i for s in range(S) for i in range(2)]
    for s, (a, b) in enumerate(pairs):
        k[2 * s + 1, 0, :2] = -1.0, -1.0 / 64
        v[2 * s, 0], v[2 * s + 1, 0] = a, -b
        z = math.log(b / a) * math.sqrt(128.0)
        q[s, 0, 0] = float(torch.tensor(z).to(torch.bfloat16))
        q[s, 0, 1] = (z - q[s, 0, 0]) * 64
    q = q.to(DEV, torch.bfloat16)
    ref.write(k, v, slots, pool)  # (all of them exact)
    table = np.full((S, W), -1)
    table[:, 0] = np.arange(S)
    out, _ = binding.cache_decode(q, to_gpu(pool), i32(table), i32([2] * S), 64, topk)
    want, _, mass = ref.decode(q.double().cpu().numpy(), pool, table, [2] * S, 64, topk)[:3]
    err = np.abs(out.double().cpu().numpy() - want)
    assert (err <= 12 * 2.0 ** -24 * mass + 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("W", WIDTHS)
@pytest.mark.parametrize("hq,hkv,topk", [(4, 1, 2), (8, 2, 3), (16, 1, 4)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_decode_nan_reaches_only_the_heads_that_attend_it(which, hq, hkv, topk, W):
    """Every past block has a NaN, which cache_write leaves for what is not finite, in a dim of
    its own; heads of a group choose different blocks, and each has the NaN of its own alone."""
    rng = np.random.default_rng(20 + topk)
    lens = [700, 64, 333]
    pool, table = some_cache(rng, lens, hkv, 64, W)
    clean = pool.copy()
    for s, L in enumerate(lens):
        for j in range((L - 1) // 64):
            at = getattr(pool, which)[table[s, j]]  # [Hkv, 64, 128] or [Hkv, 1, 128, 64]
            if which == "k":
                at[:, 3 * j, j] = 0x7f
            else:
                at[:, 0, j, 3 * j] = 0xff
    q = torch.from_numpy(rng.standard_normal((3, hq, ref.D))).to(DEV, torch.bfloat16)
    out, lse = (x.double().cpu().numpy() for x in binding.cache_decode(
        q, to_gpu(pool), i32(table), i32(lens), 64, topk))
    nq = q.double().cpu().numpy()
    want, want_lse = ref.decode(nq, pool, table, lens, 64, topk)[:2]
    bad, bad_lse = np.isnan(want), np.isnan(want_lse)
    groups = bad.reshape(3, hkv, hq // hkv, ref.D)
    assert (groups.any(2) & ~groups.all(2)).any() or which == "k"  # (heads did choose differently)
    np.testing.assert_array_equal(np.isnan(out), bad)
    np.testing.assert_array_equal(np.isnan(lse), bad_lse)
    fine = ref.decode(nq, clean, table, lens, 64, topk)  # (the same but where there is NaN)
    ref.check_decode(np.where(bad, fine[0], out), np.where(bad_lse, fine[1], lse), fine)


def far_request(length, where, fill):
    """A request of `length` tokens in a table row of 2^25 pages of 64, of which only those at
    `where` are pages of the pool; and the same pages in a row of their own, with its length.
    fill(page's place in `where`, tokens) gives its keys and values."""
    n = len(where)
    pool = ref.Pool(n + 1, 1, 64)
    near = np.arange(n)[None] + 1
    table = torch.full((2, 1 << 25), -1, dtype=torch.int32, device=DEV)
    held = 0
    for i, j in enumerate(where):
        m = min(64, length - 64 * j)
        assert m > 0 and (m == 64 or j == where[-1])
        table[0, j] = int(near[0, i])
        ref.write(*fill(i, m), near[0, i] * 64 + np.arange(m), pool)
        held += m
    return pool, table, near, held


@pytest.mark.parametrize("length", [2 ** 31 - 65, 2 ** 31 - 64, 2 ** 31 - 63, 2 ** 31 - 1])
def test_decode_lengths_up_to_32_bits(length):
    """Table rows that hold 2^31 tokens: nearly all of them are left out."""
    rng = np.random.default_rng(21)
    where = [0, 7, (1 << 24) + 5, (1 << 25) - 3, (length - 1) // 64]
    pool, table, near, held = far_request(
        length, where, lambda i, m: (rng.standard_normal((m, 1, 128)), rng.standard_normal((m, 1, 128))))
    q = torch.from_numpy(rng.standard_normal((2, 2, 128))).to(DEV, torch.bfloat16)
    out, lse = binding.cache_decode(q, to_gpu(pool), table, i32([length, 0]), 0, 0)
    want = ref.decode(q.double().cpu().numpy(), pool, np.concatenate([near, near]), [held, 0], 0, 0)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)


@pytest.mark.parametrize("length", [2 ** 31 - 64, 2 ** 31 - 1])
def test_decode_moba_lengths_up_to_32_bits(length):
    """2048 blocks of 2^20 tokens: block 3 scores above all others, which are empty but for
    block 9, which scores below them."""
    rng = np.random.default_rng(22)
    per = 1 << 14
    where = [3 * per + 1, 3 * per + 70, 9 * per, (length - 1) // 64 - 600, (length - 1) // 64]

    def fill(i, m):
        return (0.5, 0.5, -0.5, 0.5, 0.5)[i] + rng.standard_normal((m, 1, 128)), rng.standard_normal((m, 1, 128))

    pool, table, near, held = far_request(length, where, fill)
    q = torch.from_numpy(0.3 + 0.1 * rng.standard_normal((2, 2, 128))).to(DEV, torch.bfloat16)
    out, lse = binding.cache_decode(q, to_gpu(pool), table, i32([length, 0]), 1 << 20, 2)
    kept = near[:, [0, 1, 3, 4]]
    want = ref.decode(q.double().cpu().numpy(), pool, np.concatenate([kept, kept]), [held - 64, 0], 0, 0)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)


@pytest.mark.parametrize("back", [1, 64, 100, 250])
def test_cut_back_and_grown_again(back):
    """A request loses its last tokens, and the pages behind its new end go on the free list; it
    and another one grow, it is written on and decoded, both end: every page is on the list."""
    rng = np.random.default_rng(back)
    N, lens, L = 9, [300, 10], 300 - back
    pool = ref.Pool(N, 1, 64)
    cache, table, free = to_gpu(pool), i32(np.full((2, 7), -1)), i32(rng.permutation(N))
    lens_now, nf = i32([0, 0]), i32([N])
    w_table, w_free, w_lens, n = np.full((2, 7), -1), free.cpu().numpy().copy(), np.zeros(2, int), N

    def step(add, T=400):
        nonlocal w_lens, n
        p = binding.cache_plan(i32(add), lens_now, table, free, nf, 64, T, lens_out=lens_now, num_free_out=nf)
        cu, slots, w_lens, n, refused = ref.plan(add, w_lens, w_table, w_free, n, 64, T)
        np.testing.assert_array_equal(p.slots.cpu(), slots)
        np.testing.assert_array_equal(table.cpu(), w_table)
        np.testing.assert_array_equal(free.cpu(), w_free)
        assert int(nf) == n and int(p.refused) == refused == 0
        k, v = (torch.from_numpy(rng.standard_normal((T, 1, 128))).to(DEV, torch.bfloat16) for _ in range(2))
        binding.cache_write(k, v, p.slots, cache)
        ref.write(k.double().cpu().numpy(), v.double().cpu().numpy(), slots, pool)

    step(lens)
    held, gone = -(-300 // 64), -(-L // 64)
    lens_now[0] = w_lens[0] = L
    free[n:n + held - gone] = table[0, gone:held]
    w_free[n:n + held - gone] = w_table[0, gone:held]
    n += held - gone
    nf.fill_(n)
    step([90, 100])
    assert n + sum(-(-int(x) // 64) for x in w_lens) == N
    q = torch.from_numpy(rng.standard_normal((2, 2, 128))).to(DEV, torch.bfloat16)
    out, lse = binding.cache_decode(q, cache, table, lens_now, 0, 0)
    want = ref.decode(q.double().cpu().numpy(), pool, w_table, w_lens, 0, 0)
    ref.check_decode(out.double().cpu().numpy(), lse.double().cpu().numpy(), want)
    step([-1, -1])
    assert n == N and sorted(w_free[:n]) == list(range(N))


@pytest.mark.parametrize("scale", [1, 100, 2000, 10000])
@pytest.mark.parametrize("entry", [-1, -3])
def test_plan_of_a_request_whose_last_page_is_none(entry, scale):
    """A held table entry that is negative gives its tokens negative slots; the other requests,
    and the pages that this one takes, are as they would be.  Short steps, and steps whose
    slots, and whose pages, a second launch writes."""
    lens, add = [63, 127, 64, 0], [min(4, scale) if scale < 100 else 4 * scale, 3 * scale, scale, 2]
    N, T = sum(add) // 64 + 12, sum(add) + 5
    table = np.full((4, 700), -9)
    table[0, 0], table[1, :2], table[2, 0] = 0, (1, entry), 2
    rng = np.random.default_rng(scale)
    free = np.concatenate([rng.permutation(np.arange(3, N)), [0, 1, 2]])
    g_table, g_free = i32(table), i32(free)
    p = binding.cache_plan(i32(add), i32(lens), g_table, g_free, i32([N - 3]), 64, T)
    cu, slots, new, n, refused = ref.plan(add, lens, table, free, N - 3, 64, T)
    assert refused == 0 and (slots[cu[1]] < 0) and (slots[cu[1] + 1:cu[-1]] >= 0).all()
    got = p.slots.cpu().numpy()
    np.testing.assert_array_equal(np.maximum(got, -1), np.maximum(slots, -1))
    np.testing.assert_array_equal(p.cu_new.cpu(), cu)
    np.testing.assert_array_equal(p.lens.cpu(), new)
    assert int(p.num_free) == n and int(p.refused) == 0
    np.testing.assert_array_equal(g_table.cpu(), table)
    np.testing.assert_array_equal(g_free.cpu(), free)


def test_profiling_leaves_captured_calls_out():
    """A captured step while phases are timed: eager calls are counted, replays are not, and the
    calls after the count is read go on as before."""
    rng = np.random.default_rng(23)
    lens = [700, 64]
    pool, table = some_cache(rng, lens, 1, 64, 400)
    cache, t, ln = to_gpu(pool), i32(table), i32(lens)
    q = torch.randn((2, 4, 128), device=DEV).to(torch.bfloat16)
    want = binding.cache_decode(q, cache, t, ln, 64, 2)
    torch.cuda.synchronize()
    binding.profile_read()
    binding.profile_enable(True)
    try:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = binding.cache_decode(q, cache, t, ln, 64, 2)
        for _ in range(3):
            got[0].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        binding.cache_decode(q, cache, t, ln, 64, 2)
        phases = binding.profile_read()
        assert {k: n for k, (n, _) in phases.items()} == {"cache_gate": 1, "cache_attend": 1, "cache_join": 1}
    finally:
        binding.profile_enable(False)
    again = binding.cache_decode(q, cache, t, ln, 64, 2)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
