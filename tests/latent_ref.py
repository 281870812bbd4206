"""Rotary positions and latent attention in 64 bits, from their formulas, with the sums of absolute
terms that the tolerances of the GPU tests are made of."""
import math

import torch

U = 2.0 ** -8  # a rounding to bf16 is off by at most this, relative to the value
SCALE = 1.0 / math.sqrt(192.0)


def rotate(x, pos, freqs, amplitude=1.0, interleaved=False, sign=1.0):
    """x [T, H, D] -> the same in float64."""
    n = freqs.numel()
    ang = pos.double()[:, None] * freqs.double() * sign
    c, s = (ang.cos() * amplitude)[:, None], (ang.sin() * amplitude)[:, None]
    y = x.double().clone()
    i = torch.arange(n, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    y[..., a] = x.double()[..., a] * c - x.double()[..., b] * s
    y[..., b] = x.double()[..., a] * s + x.double()[..., b] * c
    return y


def rotate_bound(x, y, n, amplitude, interleaved, u):
    """Tolerance of rotate(x) = y [T, H, D].  Cosine and sine are off by at most 2^-22: the reduced angle, at
    most pi / 4, has three roundings of 2^-24 of it, the series and the amplitude as many; the
    products add two of 2^-24.  With the result's own rounding u: u |y| + 2^-21 amplitude (|x_a| + |x_b|)."""
    t = torch.zeros_like(y)
    i = torch.arange(n, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    both = x.double()[..., a].abs() + x.double()[..., b].abs()
    t[..., a] = both
    t[..., b] = both
    return u * y.abs() + 2.0 ** -21 * abs(amplitude) * t


class Attention:
    """Causal latent attention of one sequence, expanded, all in float64 [H, n, .]: out, lse; and the sums the
    tolerances need."""

    def __init__(self, q, k, kr, v, scale=SCALE):
        self.q = q.double().transpose(0, 1)
        self.k = torch.cat([k.double(), kr.double()[:, None].expand(-1, k.shape[1], -1)], 2).transpose(0, 1)
        self.v = v.double().transpose(0, 1)
        self.scale = scale
        z = self.q @ self.k.transpose(1, 2) * scale
        n = z.shape[1]
        self.mask = torch.ones((n, n), dtype=torch.bool, device=z.device).tril_()
        z = torch.where(self.mask, z, -math.inf)
        self.lse = torch.logsumexp(z, 2)
        self.p = torch.exp(z - self.lse[..., None])
        self.out = self.p @ self.v
        # largest score error of a row: fp32 sums of 192 products, each term within 2^-24 a step
        big = (self.q.abs() @ self.k.abs().transpose(1, 2)) * scale
        self.dz = torch.where(self.mask, big, 0.0).amax(2) * 192 * 2.0 ** -24 + 2.0 ** -20

    def out_bound(self):
        """Weights are rounded to bf16 (U of each) and have the error of their scores; the result is rounded."""
        c = self.p @ self.v.abs()
        return U * self.out.abs() + (U + 2 * self.dz[..., None]) * c

    def lse_bound(self):
        return self.dz + 2.0 ** -22 * self.lse.abs()

    def gradients(self, dout):
        """dq [H, n, 192], dk [H, n, 128], dkr [n, 64], dv [H, n, 128] and their tolerances, for an out and
        lse that are the GPU's own: P has U as an operand of dV; dS = P (dP - Delta) has U as an operand and,
        through the out that Delta is taken from, P times the error of <dout, out>."""
        g = dout.double().transpose(0, 1)
        dp = g @ self.v.transpose(1, 2)
        delta = (g * self.out).sum(2, keepdim=True)
        ds = self.p * (dp - delta)
        e_delta = (g.abs() * self.out_bound()).sum(2, keepdim=True)
        rel = U + 3 * self.dz[..., None]  # (score, lse and product errors)
        e_ds = rel * ds.abs() + self.p * (e_delta + 2.0 ** -16 * (g.abs() @ self.v.abs().transpose(1, 2)))
        dq, t_q = ds @ self.k * self.scale, e_ds @ self.k.abs() * self.scale
        dk, t_k = ds.transpose(1, 2) @ self.q * self.scale, e_ds.transpose(1, 2) @ self.q.abs() * self.scale
        dv = self.p.transpose(1, 2) @ g
        t_v = (rel * self.p).transpose(1, 2) @ g.abs()
        out = [dq, dk[..., :128], dk[..., 128:].sum(0), dv]
        tol = [t_q, t_k[..., :128], t_k[..., 128:].sum(0), t_v]
        return out, [t + U * x.abs() + 1e-30 for t, x in zip(tol, out)]


    def out_spread(self):
        """Variance of each result's error where every rounding to bf16 is an error of its own, at most U and
        evenly spread (U^2 / 3): of the weights as operands and of the result."""
        return U * U / 3 * (self.p ** 2 @ self.v ** 2 + self.out ** 2)

    def gradient_spread(self, dout):
        """The same of gradients(): P as the operand of dV; dS as the others', and in it Delta, whose error (of the
        forward's weights and out) all of a row's keys share; the results' roundings."""
        g = dout.double().transpose(0, 1)
        dp = g @ self.v.transpose(1, 2)
        ds = self.p * (dp - (g * self.out).sum(2, keepdim=True))
        delta = (g * self.out).square().sum(2, keepdim=True) + (self.p * dp).square().sum(2, keepdim=True)
        seen = (self.p @ self.k).square()  # (a row's error of Delta moves dq along its mean key)
        dq = (ds ** 2 @ self.k ** 2 + delta * seen) * self.scale ** 2
        dk = (ds ** 2 + self.p ** 2 * delta).transpose(1, 2) @ self.q ** 2 * self.scale ** 2
        dv = (self.p ** 2).transpose(1, 2) @ g ** 2
        want, _ = self.gradients(dout)
        return [U * U / 3 * (v + x ** 2) for v, x in
                zip((dq, dk[..., :128], dk[..., 128:].sum(0), dv), want)]


# The 2-norm of a block's errors is held to this many times the square root of their variances' sum.  Thousands of
# roundings that do not depend on each other stay close to 1 of it; a single one that outweighs all
# others is at most sqrt(3).
SPREAD = 2.0


def worst_block(got, ref, var, block=256):
    """Largest norm of errors over SPREAD times what their variances [.., n, D] ask, in each of the leading
    dims and `block` rows (the last with what is left, if that is less than a quarter)."""
    n = ref.shape[-2]
    cut = [i for i in range(0, n, block) if i == 0 or n - i >= block // 4] + [n]
    e, worst_ = (got.double() - ref).square().sum(-1), 0.0
    for i, j in zip(cut, cut[1:]):
        t = var[..., i:j, :].sum(-1).sum(-1)
        worst_ = max(worst_, float((e[..., i:j].sum(-1) / t).max()))
    return math.sqrt(worst_) / SPREAD


def decode(qc, qr, rows, scale=SCALE):
    """One request: qc [H, 512], qr [H, 64], rows [n, 576] -> out, lse and their tolerances."""
    q = torch.cat([qc, qr], 1).double()
    u = rows.double()
    z = q @ u.t() * scale
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    out = p @ u[:, :512]
    dz = (q.abs() @ u.abs().t() * scale).amax(1) * 576 * 2.0 ** -24 + 2.0 ** -20
    # the sum of the weights: fp32 terms, at most one rounding a term a lane holds
    t = U * out.abs() + (U + 2 * dz[:, None]) * (p @ u[:, :512].abs())
    return out, lse, t, dz + 2.0 ** -22 * lse.abs() + 2.0 ** -18


def worst(got, ref, tol):
    """Largest error over its tolerance."""
    return float(((got.double() - ref).abs() / tol).max()) if ref.numel() else 0.0
