"""Rotary positions on the GPU against their formula in 64 bits: layouts, partial heads, odd sizes, strides,
positions of both kinds, in place, the gradient, rows of no sequence, graphs and streams."""
import math

import pytest
import torch

import latent_ref as ref
from paper_2502_13189_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()


def randn(*shape, dtype=BF, seed=0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def check(got, x, pos, rot, sign=1.0):
    y = ref.rotate(x, pos, rot.freqs, rot.amplitude, rot.interleaved, sign)
    u = 2.0 ** -24 if x.dtype == F32 else ref.U
    tol = ref.rotate_bound(x, y, rot.freqs.numel(), rot.amplitude, rot.interleaved, u)
    assert got.dtype == x.dtype and got.shape == x.shape
    assert bool(((got.double() - y).abs() <= tol).all()), ref.worst(got, y, tol + 1e-300)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,rot", [
    (1, 1, 1, 2, 2), (1, 32, 8, 128, 128), (5, 3, 1, 64, 64), (7, 4, 2, 80, 40), (3, 5, 5, 100, 50),
    (9, 2, 1, 72, 24), (4, 1, 3, 6, 4), (33, 8, 2, 128, 64), (2, 2, 2, 7, 6), (6000, 40, 1, 64, 64),
    (3001, 31, 4, 96, 32)])
def test_rope(T, Hq, Hk, D, rot, interleaved, dtype):
    r = binding.rotation(rot, scaling="parts", factor=8.0, original_length=4096, interleaved=interleaved)
    q, k = randn(T, Hq, D, dtype=dtype, seed=1), randn(T, Hk, D, dtype=dtype, seed=2)
    pos = torch.randint(0, 1 << 20, (T,), device=DEV, dtype=torch.int32)
    qo, ko = binding.rope(q, k, r, pos=pos)
    check(qo, q, pos, r)
    check(ko, k, pos, r)
    gq, gk = binding.rope_backward(q, k, r, pos=pos)
    check(gq, q, pos, r, -1.0)
    check(gk, k, pos, r, -1.0)
    # dims that do not turn keep their bits
    assert torch.equal(qo[..., rot:], q[..., rot:]) and torch.equal(ko[..., rot:], k[..., rot:])
    # without k
    alone, none = binding.rope(q, None, r, pos=pos)
    assert none is None and torch.equal(alone, qo)
    # in place
    q2, k2 = q.clone(), k.clone()
    binding.rope(q2, k2, r, pos=pos, q_out=q2, k_out=k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("p", [0, 1, -1, 2 ** 20, -(2 ** 20), 2 ** 31 - 1, -(2 ** 31), 2 ** 40 + 12345, -(2 ** 40)])
def test_far_positions(p):
    """Angles of far positions, in whole turns taken off exactly: the reference takes them from integers."""
    freqs = torch.tensor([1.0, 0.7499, 1e-3, 1e-6, 6.5, 0.0], dtype=torch.float64)
    r = binding.Rotation(freqs.to(DEV))
    x = randn(1, 1, 12, dtype=F32, seed=3)
    pos = torch.tensor([p], dtype=torch.int64, device=DEV)
    got, _ = binding.rope(x, None, r, pos=pos)
    from fractions import Fraction
    pi = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)
    ang = []
    for f in freqs.tolist():
        t = Fraction(f) * p / (2 * pi)
        ang.append(float((t - round(t)) * 2 * pi))
    y = ref.rotate(x.cpu(), torch.ones(1), torch.tensor(ang, dtype=torch.float64))
    # a frequency's turns are held to 2^-53 of the larger of them and one turn: two roundings
    extra = abs(p) * 2.0 ** -52 * 2 * math.pi * 2
    both = x.abs().double().cpu().view(2, 6).sum(0).repeat(2)
    tol = ref.rotate_bound(x.cpu(), y, 6, 1.0, False, 2.0 ** -24) + extra * both
    assert bool(((got.cpu().double() - y).abs() <= tol).all()), ref.worst(got.cpu(), y, tol)


@pytest.mark.parametrize("p", [1, 2 ** 20, -(2 ** 20), 2 ** 31 - 1])
def test_frequencies_about_zero(p):
    """Frequencies of either sign, down to ones whose turn is lost beside 1: a whole turn less almost nothing."""
    freqs = torch.tensor([-1e-18, -1e-30, -5e-324, 1e-30, -1e-16, -1e-3, -6.5, -0.0], dtype=torch.float64)
    r = binding.Rotation(freqs.to(DEV))
    x = randn(1, 1, 16, dtype=F32, seed=4)
    got, _ = binding.rope(x, None, r, pos=torch.tensor([p], dtype=torch.int64, device=DEV))
    back, _ = binding.rope_backward(x, None, r, pos=torch.tensor([-p], dtype=torch.int64, device=DEV))
    y = ref.rotate(x, torch.tensor([p], dtype=torch.int64, device=DEV), r.freqs, 1.0, False)
    # (the reference's angles: 2^-53 of up to 6.5 p; the kernel's: 2^-52 of a turn a position)
    extra = abs(p) * (6.5 * 2.0 ** -53 + 2.0 ** -52 * 2 * math.pi)
    size = x.double().abs()
    tol = ref.rotate_bound(x, y, 8, 1.0, False, 2.0 ** -24) + extra * (size + size.roll(8, -1))
    assert bool(((got.double() - y).abs() <= tol).all()), ((got.double() - y).abs() / tol).max()
    assert bool(((back.double() - y).abs() <= tol).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_views(interleaved):
    """Parts of wider heads, heads outermost, offsets that leave rows aligned to one element only."""
    r = binding.rotation(64, interleaved=interleaved)
    pos = torch.arange(50, 50 + 37, device=DEV)
    wide = randn(37, 5, 192, seed=4)
    latent = randn(37, 576, seed=5)
    q, k = wide[:, :, 128:], latent[:, None, 512:]
    qo, ko = binding.rope(q, k, r, pos=pos)
    check(qo, q, pos, r)
    check(ko, k, pos, r)
    # in place, the rest untouched
    w2, l2 = wide.clone(), latent.clone()
    binding.rope(w2[:, :, 128:], l2[:, None, 512:], r, pos=pos, q_out=w2[:, :, 128:], k_out=l2[:, None, 512:])
    assert torch.equal(w2[..., 128:], qo) and torch.equal(l2[:, None, 512:], ko)
    assert torch.equal(w2[..., :128], wide[..., :128]) and torch.equal(l2[:, :512], latent[:, :512])
    # [H, T, D] memory, and an odd offset
    heads_first = randn(5, 37, 64, seed=6).transpose(0, 1)
    odd = randn(37, 5, 67, seed=7)[:, :, 3:]
    qo, ko = binding.rope(heads_first, odd, r, pos=pos)
    check(qo, heads_first, pos, r)
    check(ko, odd, pos, r)
    # q and k of one fused projection, in place
    fused = randn(37, 7, 64, seed=8)
    f2 = fused.clone()
    binding.rope(f2[:, :5], f2[:, 5:], r, pos=pos, q_out=f2[:, :5], k_out=f2[:, 5:])
    check(f2, fused, pos, r)


@pytest.mark.parametrize("start", [None, (7, 0, 900001, 3, 11)])
def test_sequences(start):
    """Positions from packed sequences, some empty; rows of no sequence keep what the output held."""
    r = binding.rotation(64, base=500000.0, scaling="linear", factor=4.0)
    cu = torch.tensor([2, 2, 40, 41, 41, 300], dtype=torch.int32, device=DEV)
    T = 310
    q, k = randn(T, 4, 64, seed=1), randn(T, 2, 64, seed=2)
    qo, ko = torch.full_like(q, 3.0), torch.full_like(k, 3.0)
    st = None if start is None else torch.tensor(start, dtype=torch.int32, device=DEV)
    binding.rope(q, k, r, cu_seqlens=cu, start=st, q_out=qo, k_out=ko)
    pos = torch.zeros(T, dtype=torch.int64, device=DEV)
    for s in range(5):
        a, b = int(cu[s]), int(cu[s + 1])
        pos[a:b] = torch.arange(b - a, device=DEV) + (0 if start is None else start[s])
    check(qo[2:300], q[2:300], pos[2:300], r)
    check(ko[2:300], k[2:300], pos[2:300], r)
    for x in (qo, ko):
        assert bool((x[:2] == 3.0).all()) and bool((x[300:] == 3.0).all())
    # no sequences: nothing is written
    before = qo.clone()
    binding.rope(q, None, r, cu_seqlens=cu[:1], q_out=qo)
    torch.cuda.synchronize()
    assert torch.equal(qo, before)


def test_not_finite():
    """NaN and infinities stay in their pair."""
    r = binding.rotation(64)
    q = randn(3, 2, 64, seed=9)
    bad = q.clone()
    bad[1, 1, 5], bad[2, 0, 40] = math.nan, math.inf
    pos = torch.arange(3, device=DEV)
    a, b = binding.rope(q, None, r, pos=pos)[0], binding.rope(bad, None, r, pos=pos)[0]
    same = torch.ones_like(q, dtype=torch.bool)
    same[1, 1, [5, 37]] = False
    same[2, 0, [8, 40]] = False
    assert torch.equal(a[same], b[same]) and not bool(torch.isfinite(b[~same]).any())


def test_graph_and_stream():
    """A captured step whose positions move on, replayed beside eager work; and a call on a side stream."""
    r = binding.rotation(128, interleaved=True)
    q, k = randn(64, 32, 128, seed=1), randn(64, 8, 128, seed=2)
    lens = torch.arange(64, dtype=torch.int32, device=DEV) * 100
    cu = torch.arange(65, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        qo, ko = binding.rope(q, k, r, cu_seqlens=cu, start=lens)
    torch.cuda.current_stream().wait_stream(side)
    check(qo, q, lens, r)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        qo, ko = binding.rope(q, k, r, cu_seqlens=cu, start=lens)
        lens += 1
    for _ in range(3):
        at = lens.clone()
        g.replay()
        torch.cuda.synchronize()
        check(qo, q, at, r)
        check(ko, k, at, r)
        eager, _ = binding.rope(q, k, r, cu_seqlens=cu, start=at)
        assert torch.equal(eager, qo)


def test_past_32_bits():
    """Rows beyond 2^31 elements, and strides that put them there."""
    T, H, D = 3, 2, 64
    big = torch.empty((1 << 30) * 5 // 2, dtype=BF, device=DEV)
    x = big.as_strided((T, H, D), ((1 << 30) + 64, 1 << 8, 1))
    src = randn(T, H, D, seed=3)
    x.copy_(src)
    r = binding.rotation(64)
    pos = torch.tensor([5, 6, 7], device=DEV)
    got, _ = binding.rope(x, None, r, pos=pos)
    check(got, src, pos, r)
    binding.rope(src, None, r, pos=pos, q_out=x)
    assert torch.equal(x, got)


def test_gradient_against_differences():
    """<dy, rope(x + h d) - rope(x - h d)> / 2h = <rope_backward(dy), d>: rope is linear, so any h does."""
    r = binding.rotation(32, scaling="base", factor=16.0)
    x, d, dy = (randn(11, 3, 48, dtype=F32, seed=s) for s in (1, 2, 3))
    pos = torch.arange(11, device=DEV) * 777
    up, dn = (ref.rotate(x + s * d, pos, r.freqs, r.amplitude) for s in (0.5, -0.5))
    g, _ = binding.rope_backward(dy, None, r, pos=pos)
    want, got = float(((up - dn) * dy.double()).sum()), float((g.double() * d.double()).sum())
    y = ref.rotate(dy, pos, r.freqs, r.amplitude, sign=-1.0)
    tol = float((ref.rotate_bound(dy, y, 16, r.amplitude, False, 2.0 ** -24) * d.double().abs()).sum())
    assert abs(got - want) <= tol + 1e-5  # (x + d / 2 in fp32: 2^-24 of some 1500 terms, at random)
