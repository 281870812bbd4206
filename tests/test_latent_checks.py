"""What the norms of latent attention's gradients are held to: results with the kernels' roundings are within it, results
that lack something are not.  The mistakes are planted in the 64-bit formula.  No GPU."""
import pytest
import torch

import latent_ref as ref

N, H = 640, 16
BF = torch.bfloat16
NAMES = ("dq", "dk", "dkr", "dv")


def rounded(x):
    return x.to(BF).double()


def randn(g, *shape):
    return torch.randn(shape, generator=g).to(BF)


@pytest.fixture(scope="module")
def case():
    g = torch.Generator().manual_seed(1)
    r = ref.Attention(randn(g, N, H, 192), randn(g, N, H, 128), randn(g, N, 64), randn(g, N, H, 128))
    dout = randn(g, N, H, 128)
    return r, dout, r.gradients(dout)[0], r.gradient_spread(dout)


def gradients(r, dout, p=None, late_delta=1.0, heads=slice(None), keep=None):
    """As the kernels form them: P and dS rounded to bf16 as operands, Delta from a rounded out (which rounded weights
    gave).  late_delta: factor of Delta from row 64 on; heads: those of dkr; keep: [H, N, N], what is summed."""
    g = dout.double().transpose(0, 1)
    out = rounded(rounded(r.p) @ r.v)
    factor = torch.ones((N, 1), dtype=torch.float64)
    factor[64:] = late_delta
    ds = r.p * (g @ r.v.transpose(1, 2) - factor * (g * out).sum(2, keepdim=True))
    ds, p = rounded(ds), rounded(r.p)
    if keep is not None:
        ds, p = ds * keep, p * keep
    dk = ds.transpose(1, 2) @ r.q * r.scale
    return [rounded(x) for x in (ds @ r.k * r.scale, dk[..., :128], dk[heads, :, 128:].sum(0), p.transpose(1, 2) @ g)]


def worst(case, got):
    return {n: ref.worst_block(a, x, v) for n, a, x, v in zip(NAMES, got, case[2], case[3])}


def test_roundings_are_within(case):
    r, dout = case[:2]
    w = worst(case, gradients(r, dout))
    assert max(w.values()) <= 1.0, w
    out = rounded(rounded(r.p) @ r.v)
    assert ref.worst_block(out, r.out, r.out_spread()) <= 1.0


def lost(h, rows, keys):
    keep = torch.ones((H, N, N), dtype=torch.float64)
    keep[h, rows, keys] = 0.0
    return keep


@pytest.mark.parametrize("name,plant,seen", [
    ("a head of dkr", dict(heads=slice(0, H - 1)), ("dkr",)),
    ("Delta from row 64 on", dict(late_delta=0.0), ("dq", "dk", "dkr")),
    ("a tile of a head", dict(keep=lost(3, slice(448, 512), slice(128, 192))), NAMES),
    ("the last rows' tile", dict(keep=lost(3, slice(576, 640), slice(0, 64))), NAMES),
    ("a tile on the diagonal", dict(keep=lost(3, slice(320, 384), slice(320, 384))), NAMES),
    ("rows from 256 on for a block of keys", dict(keep=lost(slice(None), slice(256, N), slice(128, 256))), NAMES)])
def test_mistakes_are_seen(case, name, plant, seen):
    w = worst(case, gradients(*case[:2], **plant))
    assert all(w[n] > 1.0 for n in seen), (name, w)


def test_blocks():
    """Whole blocks, and what is left over with the last of them or by itself."""
    x = torch.zeros((1, 600, 2), dtype=torch.float64)
    for at in (0, 255, 256, 511, 512, 599):
        y = x.clone()
        y[0, at, 1] = 1.0
        n = 256 if at < 512 else 88
        assert abs(ref.worst_block(y, x, x + 1.0) * ref.SPREAD - (1 / (2 * n)) ** 0.5) < 1e-12, at
    y = x[:, :300].clone()
    y[0, 299, 0] = 1.0
    assert abs(ref.worst_block(y, x[:, :300], x[:, :300] + 1.0) * ref.SPREAD - (1 / 600) ** 0.5) < 1e-12
