"""Latent attention on the GPU against its formulas in 64 bits: the expanded form and its gradients, the paged
cache's write and decode, and runs of them together."""
import math

import pytest
import torch

import latent_ref as ref
from paper_2502_13189_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()


def randn(*shape, seed=0, size=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * size).to(BF)


def cu_of(lens, first=0):
    cu = [first]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=DEV)


def inputs(T, H, seed=0, size=1.0):
    """q, k, k_rope, v: k and v views of one projection, k_rope of the latent rows."""
    kv = randn(T, H, 256, seed=seed + 1)
    return (randn(T, H, 192, seed=seed, size=size), kv[..., :128], randn(T, 576, seed=seed + 2)[:, 512:],
            kv[..., 128:])


def check_forward(q, k, kr, v, cu, out, lse, scale=ref.SCALE):
    for a, b in zip(cu.tolist(), cu.tolist()[1:]):
        if a == b:
            continue
        r = ref.Attention(q[a:b], k[a:b], kr[a:b], v[a:b], scale)
        w = ref.worst(out[a:b].transpose(0, 1), r.out, r.out_bound())
        assert w <= 1.0, (a, b, w)
        w = ref.worst(lse[:, a:b], r.lse, r.lse_bound())
        assert w <= 1.0, (a, b, "lse", w)


def check_backward(q, k, kr, v, cu, dout, grads, scale=ref.SCALE):
    dq, dk, dkr, dv = grads
    for a, b in zip(cu.tolist(), cu.tolist()[1:]):
        if a == b:
            continue
        want, tol = ref.Attention(q[a:b], k[a:b], kr[a:b], v[a:b], scale).gradients(dout[a:b])
        got = (dq[a:b].transpose(0, 1), dk[a:b].transpose(0, 1), dkr[a:b], dv[a:b].transpose(0, 1))
        for name, g, x, t in zip(("dq", "dk", "dkr", "dv"), got, want, tol):
            w = ref.worst(g, x, t)
            assert w <= 1.0, (name, a, b, w)


LENS = [((1,), 1), ((2, 1, 0, 63), 3), ((64, 65, 0, 1), 5), ((127, 128, 129), 8), ((255, 256, 257, 31), 2),
        ((700, 1, 333), 4), ((1023,), 10), ((33,) * 20, 1), ((2049, 65), 1)]


@pytest.mark.parametrize("lens,H", LENS)
def test_forward(lens, H):
    q, k, kr, v = inputs(sum(lens), H, seed=sum(lens))
    cu = cu_of(lens)
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    check_forward(q, k, kr, v, cu, out, lse)
    again, lse2 = binding.latent_forward(q, k, kr, v, cu)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("lens,H", LENS)
def test_backward(lens, H):
    q, k, kr, v = inputs(sum(lens), H, seed=sum(lens))
    cu = cu_of(lens)
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    dout = randn(sum(lens), H, 128, seed=77)
    grads = binding.latent_backward(q, k, kr, v, cu, out, lse, dout)
    check_backward(q, k, kr, v, cu, dout, grads)
    for x, y in zip(grads, binding.latent_backward(q, k, kr, v, cu, out, lse, dout)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("lens,H", [
    (tuple(37 * i % 301 for i in range(63)) + (700,), 3), (tuple(37 * i % 301 for i in range(64)) + (700,), 3),
    ((1100, 30), 100), ((1100, 30), 110), ((200, 55), 2), ((200, 56), 2), ((0, 0, 513, 0), 2)])
def test_backward_launches(lens, H):
    """About the limits up to which both sides share a launch: 64 sequences, of 128 tokens on average, 1024 work-groups
    a side; the forward's work-groups, ranked or not."""
    q, k, kr, v = inputs(sum(lens), H, seed=sum(lens))
    cu = cu_of(lens)
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    check_forward(q, k, kr, v, cu, out, lse)
    dout = randn(sum(lens), H, 128, seed=78)
    check_backward(q, k, kr, v, cu, dout, binding.latent_backward(q, k, kr, v, cu, out, lse, dout))


@pytest.mark.parametrize("size,scale", [(8.0, ref.SCALE), (0.01, 1.0), (3.0, 0.3)])
def test_scores_of_other_sizes(size, scale):
    """Peaked and flat softmax: the running max moves often, or never."""
    q, k, kr, v = inputs(500, 3, seed=5, size=size)
    cu = cu_of((500,))
    out, lse = binding.latent_forward(q, k, kr, v, cu, scale=scale)
    check_forward(q, k, kr, v, cu, out, lse, scale)
    dout = randn(500, 3, 128, seed=6)
    check_backward(q, k, kr, v, cu, dout, binding.latent_backward(q, k, kr, v, cu, out, lse, dout, scale=scale), scale)


def test_rising_scores():
    """Every key outweighs those before it by far, so that every tile raises the max."""
    T, H = 400, 2
    q, k, kr, v = inputs(T, H, seed=9)
    k = k.clone()
    q[..., 0] = 8.0
    k[..., 0] = (torch.arange(T, device=DEV) * 0.5)[:, None].to(BF)
    cu = cu_of((T,))
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    check_forward(q, k, kr, v, cu, out, lse)


def test_padded_batch():
    """Rows outside the sequences keep what the outputs held."""
    T, H = 300, 3
    q, k, kr, v = inputs(T, H)
    cu = cu_of((100, 0, 61), first=5)
    for x in (q, kr):  # (what stands there is never used)
        x[:5], x[166:] = math.nan, math.nan
    out, lse = torch.full((T, H, 128), 3.0, dtype=BF, device=DEV), torch.full((H, T), 3.0, device=DEV)
    binding.latent_forward(q, k, kr, v, cu, out=out, lse=lse)
    check_forward(q, k, kr, v, cu, out, lse)
    dout = randn(T, H, 128, seed=3)
    grads = [torch.full_like(x, 3.0, memory_format=torch.contiguous_format) for x in (q, k, kr, v)]
    binding.latent_backward(q, k, kr, v, cu, out, lse, dout, dq=grads[0], dk=grads[1], dk_rope=grads[2], dv=grads[3])
    check_backward(q, k, kr, v, cu, dout, grads)
    for x in (out, *grads, lse.t()):
        assert bool((x[:5] == 3.0).all()) and bool((x[166:] == 3.0).all())


def test_views():
    """Heads outermost, gradients into one projection's memory."""
    T, H = 130, 3
    q = randn(H, T, 192).transpose(0, 1)
    _, k, kr, v = inputs(T, H, seed=4)
    cu = cu_of((70, 60))
    out = torch.empty((H, T, 128), dtype=BF, device=DEV).transpose(0, 1)
    _, lse = binding.latent_forward(q, k, kr, v, cu, out=out)
    check_forward(q, k, kr, v, cu, out, lse)
    dout = randn(T, H, 128, seed=8)
    dkv, dc = torch.empty((T, H, 256), dtype=BF, device=DEV), torch.zeros((T, 576), dtype=BF, device=DEV)
    grads = binding.latent_backward(q, k, kr, v, cu, out, lse, dout, dk=dkv[..., :128], dv=dkv[..., 128:],
                                    dk_rope=dc[:, 512:])
    check_backward(q, k, kr, v, cu, dout, grads)
    assert not bool(dc[:, :512].any())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_not_finite_values_stay_with_those_who_attend(bad):
    T, H = 200, 2
    q, k, kr, v = inputs(T, H, seed=2)
    cu = cu_of((150, 50))
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    v2, k2 = v.clone(), k.clone()
    v2[100, 1, 7] = bad       # a row before it does not see it
    v2[149, 0, 3] = bad       # the sequence's last: its tile repeats it past the end
    k2[140, 1] = bad
    out2, lse2 = binding.latent_forward(q, k2, kr, v2, cu)
    same = torch.ones_like(out, dtype=torch.bool)
    same[100:150, 1, 7] = False
    same[149, 0, 3] = False
    same[140:150, 1] = False
    # such a tile's keys are summed one by one: another order of the same fp32 terms, so the results agree not
    # to the bit, but each is within the formula's tolerance, which holds for any order
    assert bool(torch.isfinite(out2[same]).all())
    check_forward(q, k, kr, v, cu, torch.where(same, out2, out), lse)
    want = out2[100:140, 1, 7]
    assert bool(torch.isnan(want).all() if math.isnan(bad) else (want == bad).all())
    assert not math.isfinite(float(out2[149, 0, 3]))
    assert torch.equal(lse[0], lse2[0]) and torch.equal(lse[1, :140], lse2[1, :140])
    assert torch.equal(lse[1, 150:], lse2[1, 150:])


def test_gradient_against_differences():
    """<dout, out(x + h d) - out(x - h d)> / 2h against the gradients along d, out in 64 bits."""
    T, H = 90, 2
    q, k, kr, v = inputs(T, H, seed=3)
    cu = cu_of((T,))
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    dout = randn(T, H, 128, seed=5)
    grads = binding.latent_backward(q, k, kr, v, cu, out, lse, dout)
    _, tol = ref.Attention(q, k, kr, v).gradients(dout)
    tol = [t.transpose(0, 1) if t.dim() == 3 else t for t in tol]
    xs = [x.double() for x in (q, k, kr, v)]
    h = 1e-4
    for i in range(4):
        d = randn(*xs[i].shape, seed=20 + i).double()
        loss = []
        for s in (h, -h):
            y = list(xs)
            y[i] = xs[i] + s * d
            loss.append(float((ref.Attention(*y).out.transpose(0, 1) * dout.double()).sum()))
        want = (loss[0] - loss[1]) / (2 * h)
        got = float((grads[i].double() * d).sum())
        # (the differences' own error: h^2 of third derivatives, and 2^-52 of sums of some 10^4 terms over h)
        assert abs(got - want) <= float((tol[i] * d.abs()).sum()) + 1e-4, i


def test_far_rows():
    """Token strides that put rows beyond 2^31 elements; inputs, outputs and gradients apart in one buffer."""
    T, H, st = 300, 2, 1 << 23
    big = torch.empty(T * st, dtype=BF, device=DEV)
    q, k, kr, v = inputs(T, H, seed=6)
    dout = randn(T, H, 128, seed=7)
    cu = cu_of((299, 1))

    def place(x, at):
        y = big.as_strided(x.shape, (st, 192, 1) if x.dim() == 3 else (st, 1), at)
        y.copy_(x)
        return y

    q2, k2, v2, kr2, g2 = place(q, 0), place(k, 512), place(v, 1024), place(kr, 1536), place(dout, 2048)
    blank = lambda x, at: place(torch.zeros_like(x, memory_format=torch.contiguous_format), at)  # noqa: E731
    out, dq, dk, dv, dkr = (blank(x, 2560 + 512 * i) for i, x in enumerate((v, q, k, v, kr)))
    _, lse = binding.latent_forward(q2, k2, kr2, v2, cu, out=out)
    check_forward(q, k, kr, v, cu, out, lse)
    grads = binding.latent_backward(q2, k2, kr2, v2, cu, out, lse, g2, dq=dq, dk=dk, dk_rope=dkr, dv=dv)
    check_backward(q, k, kr, v, cu, dout, grads)


def test_side_streams():
    """Calls on several streams at once, outputs and workspaces allocated for the stream of their call."""
    lens, H = (150, 333), 3
    T = sum(lens)
    sets = [(*inputs(T, H, seed=10 * i), randn(T, H, 128, seed=10 * i + 5)) for i in range(3)]
    cu = cu_of(lens)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for (q, k, kr, v, dout), st in zip(sets, streams):
        for _ in range(4):
            out, lse = binding.latent_forward(q, k, kr, v, cu, stream=st)
            grads = binding.latent_backward(q, k, kr, v, cu, out, lse, dout, stream=st)
        got.append((out, lse, *grads))
    torch.cuda.synchronize()
    for (q, k, kr, v, dout), x in zip(sets, got):
        out, lse = binding.latent_forward(q, k, kr, v, cu)
        for a, b in zip(x, (out, lse, *binding.latent_backward(q, k, kr, v, cu, out, lse, dout))):
            assert torch.equal(a, b)


def test_backward_workspace():
    """A workspace of the exact size, holding NaN; one too small is refused."""
    T, H = 100, 3
    q, k, kr, v = inputs(T, H)
    cu, dout = cu_of((60, 40)), randn(T, H, 128, seed=5)
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    want = binding.latent_backward(q, k, kr, v, cu, out, lse, dout)
    need = binding.latent_backward_workspace_bytes(T, H)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    for _ in range(2):
        for a, b in zip(want, binding.latent_backward(q, k, kr, v, cu, out, lse, dout, workspace=ws)):
            assert torch.equal(a, b)
    with pytest.raises(binding.MobaError, match="NO_MEMORY"):
        binding.latent_backward(q, k, kr, v, cu, out, lse, dout, workspace=ws[:need - 1])


def test_long_sequences():
    """The forward's work-groups of 256 queries (many long sequences): rows of each of them."""
    T, H = 8300, 33
    q, k, kr, v = inputs(T, H, seed=8)
    cu = cu_of((T,))
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    for h in (0, 17, 32):
        r = ref.Attention(q[:, h:h + 1], k[:, h:h + 1], kr, v[:, h:h + 1])
        assert ref.worst(out[:, h:h + 1].transpose(0, 1), r.out, r.out_bound()) <= 1.0
        assert ref.worst(lse[h:h + 1], r.lse, r.lse_bound()) <= 1.0


def test_graph_of_forward_and_backward():
    """Captured together, replayed on new inputs beside eager calls of the same shapes."""
    lens, H = (200, 57), 3
    T = sum(lens)
    q, k, kr, v = inputs(T, H)
    dout, cu = randn(T, H, 128, seed=6), cu_of(lens)
    binding.latent_backward(q, k, kr, v, cu, *binding.latent_forward(q, k, kr, v, cu), dout)  # warm
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out, lse = binding.latent_forward(q, k, kr, v, cu)
        grads = binding.latent_backward(q, k, kr, v, cu, out, lse, dout)
    for s in range(3):
        q.copy_(randn(T, H, 192, seed=30 + s))
        cu.copy_(cu_of((200 - s, 57 + s)))
        g.replay()
        torch.cuda.synchronize()
        o2, l2 = binding.latent_forward(q, k, kr, v, cu)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        for x, y in zip(grads, binding.latent_backward(q, k, kr, v, cu, o2, l2, dout)):
            assert torch.equal(x, y)


# ------------------------------------------------------------------- paged cache
def paged(lens, page, seed=0, extra=3, fill=None):
    """pages with the requests' rows (what lies behind them: `fill`, or NaN), table, lens, the rows."""
    held = [-(-n // page) for n in lens]
    N = sum(held) + extra
    pages = torch.full((N, page, 576), math.nan if fill is None else fill, dtype=BF, device=DEV)
    ids = torch.randperm(N, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), max(max(held), 1)), N + 7, dtype=torch.int32, device=DEV)
    rows = []
    for s, n in enumerate(lens):
        x = randn(n, 576, seed=seed * 1000 + s)
        for j in range(held[s]):
            at = ids.pop()
            table[s, j] = at
            part = x[j * page:(j + 1) * page]
            pages[at, :part.shape[0]] = part
        rows.append(x)
    return pages, table, torch.tensor(lens, dtype=torch.int32, device=DEV), rows


def check_decode(qc, qr, rows, out, lse, scale=ref.SCALE):
    for s, u in enumerate(rows):
        if not u.shape[0]:
            assert not bool(out[s].any()) and bool((lse[:, s] == -math.inf).all())
            continue
        o, l, to, tl = ref.decode(qc[s], qr[s], u, scale)
        assert ref.worst(out[s], o, to) <= 1.0, (s, u.shape[0], ref.worst(out[s], o, to))
        assert ref.worst(lse[:, s], l, tl) <= 1.0, (s, u.shape[0], "lse")


@pytest.mark.parametrize("H", [1, 5, 16, 17, 32, 40, 64, 128])
@pytest.mark.parametrize("lens,page", [((1,), 64), ((700, 333, 0), 64), ((0, 64, 65, 63, 0, 128, 1, 0), 128),
                                       ((5000,), 192), ((1, 20011, 0, 300, 256, 257), 256)])
def test_decode(lens, page, H):
    pages, table, ln, rows = paged(lens, page, seed=H)
    qc, qr = randn(len(lens), H, 512, seed=1), randn(len(lens), H, 192, seed=2)[..., 128:]
    out, lse = binding.latent_decode(qc, qr, pages, table, ln)
    check_decode(qc, qr, rows, out, lse)
    out2, lse2 = binding.latent_decode(qc, qr, pages, table, ln)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("H", [17, 33, 40, 64, 128, 130])
@pytest.mark.parametrize("lens,page", [((1,), 64), ((700, 333, 0), 64), ((0, 64, 65, 63, 0, 128, 1, 0), 128),
                                       ((5000,), 192), ((1, 20011, 0, 300, 256, 257), 256)])
def test_decode_wide_tables(lens, page, H):
    """Tables far wider than the requests, as a captured step has them: the heads go in the largest groups."""
    pages, table, ln, rows = paged(lens, page, seed=H)
    more = -(-(1 << 24) // (len(lens) * page * H))
    table = torch.cat([table, torch.full((len(lens), more), -1, dtype=torch.int32, device=DEV)], 1)
    qc, qr = randn(len(lens), H, 512, seed=1), randn(len(lens), H, 64, seed=2)
    out, lse = binding.latent_decode(qc, qr, pages, table, ln)
    check_decode(qc, qr, rows, out, lse)


@pytest.mark.parametrize("H", [8, 20, 128])
def test_decode_many_requests(H):
    """More requests than work-groups, many in one run, some split over two."""
    lens = [(i * 37) % 200 if i % 7 else 0 for i in range(600)] + [9000]
    pages, table, ln, rows = paged(lens, 64, seed=1)
    qc, qr = randn(len(lens), H, 512, seed=1), randn(len(lens), H, 64, seed=2)
    out, lse = binding.latent_decode(qc, qr, pages, table, ln, scale=0.1)
    check_decode(qc, qr, rows, out, lse, 0.1)


def test_decode_lengths_on_the_edge():
    """Lengths below 0 and past the table count as 0 and its end; entries of no page are masked, at any place."""
    pages, table, ln, rows = paged((300, 200, 130, 64, 128), 64)
    qc, qr = randn(5, 8, 512, seed=1), randn(5, 8, 64, seed=2)
    table = table.clone()
    ln = torch.tensor([100000, -5, 130, 64, 128], dtype=torch.int32, device=DEV)
    pages[table[0, 4].long(), 44:] = pages[0, :20] * 0 + 1.0  # (the last page is full then)
    rows[0] = torch.cat([rows[0], torch.ones((20, 576), dtype=BF, device=DEV)])
    rows[1] = rows[1][:0]
    table[2, 1], table[3, 0] = -3, 1 << 30
    rows[2] = torch.cat([rows[2][:64], rows[2][128:]])
    rows[3] = rows[3][:0]
    table[4, 0] = 2 ** 31 - 1
    rows[4] = rows[4][64:]
    out, lse = binding.latent_decode(qc, qr, pages, table, ln)
    check_decode(qc, qr, rows, out, lse)


def test_decode_rising_scores():
    """Later tokens outweigh earlier ones by far: the running max is raised step by step."""
    n, H = 1000, 40
    pages, table, ln, rows = paged((n,), 64)
    u = rows[0]
    u[:, 0] = torch.arange(n, device=DEV).to(BF)
    for j in range(-(-n // 64)):
        part = u[j * 64:(j + 1) * 64]
        pages[table[0, j].long(), :part.shape[0]] = part
    qc, qr = randn(1, H, 512, seed=1), randn(1, H, 64, seed=2)
    qc[..., 0] = torch.linspace(-8, 8, H, device=DEV).to(BF)
    out, lse = binding.latent_decode(qc, qr, pages, table, ln)
    check_decode(qc, qr, rows, out, lse)


def test_decode_not_finite():
    """NaN in a request stays there."""
    pages, table, ln, rows = paged((300, 200, 130), 64)
    qc, qr = randn(3, 8, 512, seed=1), randn(3, 8, 64, seed=2)
    out, lse = binding.latent_decode(qc, qr, pages, table, ln)
    pages[table[1, 1].long(), 5, 9] = math.nan
    out2, lse2 = binding.latent_decode(qc, qr, pages, table, ln)
    for s in (0, 2):
        assert torch.equal(out[s], out2[s]) and torch.equal(lse[:, s], lse2[:, s])
    assert bool(torch.isnan(out2[1]).all())


def test_decode_far_pages():
    """Pages beyond 2^31 elements of the pool."""
    P = 64
    N = (1 << 31) // (P * 576) + 50
    pages = torch.empty((N, P, 576), dtype=BF, device=DEV)
    u = randn(100, 576)
    pages[N - 1], pages[N - 2, :36] = u[:64], u[64:]
    table = torch.tensor([[N - 1, N - 2]], dtype=torch.int32, device=DEV)
    ln = torch.tensor([100], dtype=torch.int32, device=DEV)
    qc, qr = randn(1, 8, 512, seed=1), randn(1, 8, 64, seed=2)
    out, lse = binding.latent_decode(qc, qr, pages, table, ln)
    check_decode(qc, qr, [u], out, lse)
    slots = torch.tensor([(N - 3) * P + 5], device=DEV)
    binding.latent_write(u[:1, :512], u[:1, 512:], slots, pages)
    assert torch.equal(pages[N - 3, 5], u[0])


def test_decode_workspace():
    """A workspace of the exact size serves calls one after the other and two graphs; one too small is refused."""
    pages, table, ln, rows = paged((900, 70), 64)
    qc, qr = randn(2, 20, 512, seed=1), randn(2, 20, 64, seed=2)
    need = binding.latent_decode_workspace_bytes(2, table.shape[1], 20, 64)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
    want, wl = binding.latent_decode(qc, qr, pages, table, ln)
    out, lse = binding.latent_decode(qc, qr, pages, table, ln, workspace=ws)
    assert torch.equal(out, want) and torch.equal(lse, wl)
    with pytest.raises(binding.MobaError, match="NO_MEMORY"):
        binding.latent_decode(qc, qr, pages, table, ln, workspace=ws[:need - 1])
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = binding.latent_decode(qc, qr, pages, table, ln, workspace=ws)
        graphs.append((g, res))
    for n in (900, 5, 64):
        ln[0] = n
        want, wl = binding.latent_decode(qc, qr, pages, table, ln)
        for g, (o, l) in graphs:
            o.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want) and torch.equal(l, wl)


@pytest.mark.parametrize("interleaved", [False, True])
def test_write(interleaved):
    r = binding.rotation(64, interleaved=interleaved, scaling="parts", factor=8.0, original_length=4096)
    T, P = 333, 128
    pages = torch.full((6, P, 576), 7.0, dtype=BF, device=DEV)
    c, kr = randn(T, 576, seed=1)[:, :512], randn(T, 192, seed=2)[:, 128:]
    slots = torch.randperm(6 * P, generator=torch.Generator().manual_seed(1))[:T].to(DEV)
    slots[5], slots[9], slots[200] = -1, 6 * P, -(2 ** 40)
    pos = torch.randint(0, 1 << 20, (T,), device=DEV)
    plain = pages.clone()
    binding.latent_write(c, kr, slots, plain)
    binding.latent_write(c, kr, slots, pages, r, pos=pos)
    ok = (slots >= 0) & (slots < 6 * P)
    flat, pflat = pages.view(-1, 576), plain.view(-1, 576)
    assert torch.equal(flat[slots[ok]][:, :512], c[ok]) and torch.equal(pflat[slots[ok]], torch.cat([c, kr], 1)[ok])
    y = ref.rotate(kr[:, None], pos, r.freqs, r.amplitude, interleaved)
    tol = ref.rotate_bound(kr[:, None], y, 32, r.amplitude, interleaved, ref.U)
    assert ref.worst(flat[slots[ok]][:, 512:], y[ok, 0], tol[ok, 0] + 1e-300) <= 1.0
    # the same as rope() gives
    assert torch.equal(flat[slots[ok]][:, 512:], binding.rope(kr[:, None], None, r, pos=pos)[0][ok, 0])
    rest = torch.ones(6 * P, dtype=torch.bool, device=DEV)
    rest[slots[ok]] = False
    assert bool((flat[rest] == 7.0).all()) and bool((pflat[rest] == 7.0).all())


def test_write_by_sequences():
    """Positions from packed sequences; a row of no sequence is left out though it has a slot."""
    r = binding.rotation(64)
    T = 21
    c, kr = randn(T, 512, seed=1), randn(T, 64, seed=2)
    pages = torch.full((2, 64, 576), 7.0, dtype=BF, device=DEV)
    cu = torch.tensor([2, 12, 12, 19], dtype=torch.int32, device=DEV)
    start = torch.tensor([5, 0, 1000], dtype=torch.int32, device=DEV)
    slots = torch.arange(T, device=DEV) + 50
    binding.latent_write(c, kr, slots, pages, r, cu_seqlens=cu, start=start)
    pos = torch.cat([torch.arange(5, 15, device=DEV), torch.arange(1000, 1007, device=DEV)])
    want = torch.full((128, 576), 7.0, dtype=BF, device=DEV)
    want[52:69] = torch.cat([c[2:19], binding.rope(kr[2:19, None], None, r, pos=pos)[0][:, 0]], 1)
    assert torch.equal(pages.view(-1, 576), want)
    binding.latent_write(c, kr, slots, pages, r, cu_seqlens=cu[:1])
    torch.cuda.synchronize()
    assert torch.equal(pages.view(-1, 576), want)


def test_write_page_stride():
    """A layer's slice of a pool of several layers."""
    pool = torch.full((4, 3, 64, 576), 7.0, dtype=BF, device=DEV)
    c, kr = randn(10, 512), randn(10, 64)
    slots = torch.arange(60, 70, device=DEV)
    binding.latent_write(c, kr, slots, pool[:, 1])
    assert torch.equal(pool[:, 1].reshape(-1, 576)[slots], torch.cat([c, kr], 1))
    assert bool((pool[:, 0] == 7.0).all()) and bool((pool[:, 2] == 7.0).all())
    table = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV)
    pool[:, 1].view(4, -1, 576)[0, :60] = randn(60, 576, seed=3)
    ln = torch.tensor([70], dtype=torch.int32, device=DEV)
    qc, qr = randn(1, 4, 512, seed=1), randn(1, 4, 64, seed=2)
    out, lse = binding.latent_decode(qc, qr, pool[:, 1], table, ln)
    check_decode(qc, qr, [pool[:2, 1].reshape(-1, 576)[:70]], out, lse)


# ------------------------------------------------------------------- together
def test_serving_run():
    """A captured serving step (plan, rotary positions, write, decode) replayed while requests come, grow and
    go; every replay against the formula over all that was fed."""
    S, P, N, H, W = 4, 64, 40, 12, 6
    r = binding.rotation(64, interleaved=True)
    pages = binding.latent_cache_new(N, P)
    pages.fill_(math.nan)
    i32 = dict(dtype=torch.int32, device=DEV)
    table, lens, add = torch.zeros((S, W), **i32), torch.zeros(S, **i32), torch.zeros(S, **i32)
    free, nfree = torch.arange(N, **i32), torch.tensor([N], **i32)
    T = 200
    c, kr = torch.zeros((T, 512), dtype=BF, device=DEV), torch.zeros((T, 64), dtype=BF, device=DEV)
    qc, q = torch.zeros((S, H, 512), dtype=BF, device=DEV), torch.zeros((S, H, 192), dtype=BF, device=DEV)

    def step():
        before = lens.clone()
        plan = binding.cache_plan(add, lens, table, free, nfree, P, T, lens_out=lens, num_free_out=nfree)
        binding.latent_write(c, kr, plan.slots, pages, r, cu_seqlens=plan.cu_new, start=before)
        qr, _ = binding.rope(q[..., 128:], None, r, pos=lens - 1)
        return binding.latent_decode(qc, qr, pages, table, lens)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = step()
    held = [[] for _ in range(S)]
    for n, adds in enumerate([(100, 3, 0, 64), (1, 1, 64, 1), (1, -1, 1, 1), (30, 70, 1, -1), (1, 1, 1, 90)]):
        add.copy_(torch.tensor(adds, **i32))
        c.copy_(randn(T, 512, seed=n))
        kr.copy_(randn(T, 64, seed=100 + n))
        qc.copy_(randn(S, H, 512, seed=200 + n))
        q.copy_(randn(S, H, 192, seed=300 + n))
        g.replay()
        torch.cuda.synchronize()
        at = 0
        for s, a in enumerate(adds):
            if a < 0:
                held[s] = []
                continue
            pos = torch.arange(len(held[s]), len(held[s]) + a, device=DEV)
            turned = binding.rope(kr[at:at + a, None], None, r, pos=pos)[0][:, 0]
            held[s] += list(torch.cat([c[at:at + a], turned], 1))
            at += a
        ln = torch.tensor([len(x) for x in held], device=DEV)
        assert lens.tolist() == ln.tolist()
        qr = binding.rope(q[..., 128:], None, r, pos=ln - 1)[0]
        check_decode(qc, qr, [torch.stack(x) if x else c[:0, :1].expand(0, 576) for x in held], out, lse)


def test_absorbed_equals_expanded():
    """Decode over the cache gives the expanded form's last row: the query folded by the keys' projection, the
    result projected to values; compared through the 64-bit formula of each side's own bf16 inputs."""
    T, H = 333, 4
    r = binding.rotation(64)
    wk, wv = randn(H, 128, 512, seed=1, size=0.05), randn(H, 128, 512, seed=2, size=0.05)
    c, kr, q = randn(T, 512, seed=3), randn(T, 64, seed=4), randn(T, H, 192, seed=5)
    pos, cu = torch.arange(T, device=DEV), cu_of((T,))
    k = torch.einsum("tr,hdr->thd", c.float(), wk.float()).to(BF)
    v = torch.einsum("tr,hdr->thd", c.float(), wv.float()).to(BF)
    q2 = q.clone()
    _, kr2 = binding.rope(q2[..., 128:], kr[:, None], r, pos=pos, q_out=q2[..., 128:])
    out, lse = binding.latent_forward(q2, k, kr2[:, 0], v, cu)
    pages = binding.latent_cache_new(6)
    table = torch.randperm(6, generator=torch.Generator().manual_seed(2)).to(torch.int32).to(DEV)[None]
    slots = table[0][pos // 64].long() * 64 + pos % 64
    binding.latent_write(c, kr, slots, pages, r, pos=pos)
    qc = torch.einsum("hd,hdr->hr", q[-1, :, :128].float(), wk.float())[None]
    o2, l2 = binding.latent_decode(qc.to(BF), q2[-1:, :, 128:], pages, table, torch.tensor([T], dtype=torch.int32, device=DEV))
    got = torch.einsum("hr,hdr->hd", o2[0].double(), wv.double())
    # what separates the two: k and v rounded to bf16 (a score: 128 products, U each of |q| |k|), the
    # folded query (512 of U |qc| |c|), and the two results' own roundings
    a = ref.Attention(q2, k, kr2[:, 0], v)
    z1 = (q[-1, :, :128].double().abs()[:, None] * k.double().abs().transpose(0, 1)).sum(2).amax(1)
    z2 = (qc[0].double().abs()[:, None] * c.double().abs()[None]).sum(2).amax(1)
    dz = (ref.U * (z1 + z2)) * ref.SCALE + a.dz[:, -1]
    assert bool(((lse[:, -1].double() - l2[:, 0].double()).abs() <= dz).all())
    cv = (a.p[:, -1:] @ a.v.abs())[:, 0]
    co = torch.einsum("hr,hdr->hd", o2[0].double().abs(), wv.double().abs())
    tol = 2 * ref.U * cv + 2 * ref.U * co + (torch.exp(2 * dz) - 1)[:, None] * cv
    assert bool(((out[-1].double() - got).abs() <= tol).all())


def test_training_chain():
    """Rotary positions, latent attention and both gradients, against differences of the formula's loss."""
    T, H = 70, 2
    r = binding.rotation(64, interleaved=True)
    q, k, kr, v = inputs(T, H, seed=11)
    pos, cu = torch.arange(T, device=DEV) + 1000, cu_of((T,))
    q2, kr2 = q.clone(), kr[:, None].clone()
    binding.rope(q2[..., 128:], kr2, r, pos=pos, q_out=q2[..., 128:], k_out=kr2)
    out, lse = binding.latent_forward(q2, k, kr2[:, 0], v, cu)
    dout = randn(T, H, 128, seed=12)
    dq, dk, dkr, dv = binding.latent_backward(q2, k, kr2[:, 0], v, cu, out, lse, dout)
    _, tol = ref.Attention(q2, k, kr2[:, 0], v).gradients(dout)
    binding.rope_backward(dq[..., 128:], dkr[:, None], r, pos=pos, dq=dq[..., 128:], dk=dkr[:, None])

    def loss(xq, xkr):
        y = xq.clone()
        y[..., 128:] = ref.rotate(xq[..., 128:], pos, r.freqs, 1.0, True)
        return float((ref.Attention(y, k.double(), ref.rotate(xkr[:, None], pos, r.freqs, 1.0, True)[:, 0],
                                    v.double()).out.transpose(0, 1) * dout.double()).sum())

    h = 1e-4
    for i, (g, t) in enumerate(((dq, tol[0].transpose(0, 1)), (dkr, tol[2]))):
        x = [q.double(), kr.double()]
        d = randn(*x[i].shape, seed=30 + i).double()
        up, dn = list(x), list(x)
        up[i], dn[i] = x[i] + h * d, x[i] - h * d
        want, got = (loss(*up) - loss(*dn)) / (2 * h), float((g.double() * d).sum())
        # turned inputs rounded to bf16 move the point the gradient is taken at: U of it, and of the gradient,
        # besides the tolerance; a turn mixes pairs, so their tolerances add (factor 2)
        scale = float((g.double().abs() * d.abs()).sum())
        assert abs(got - want) <= 2 * float((t * d.abs()).sum()) + 2 * ref.U * scale + 1e-4, i
