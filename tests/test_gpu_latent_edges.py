"""Latent attention on the GPU where a call is largest: the limits of its launches."""
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


def randn(*shape, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(BF)


def test_decode_of_two_million_requests():
    """One head: the join's work-groups, eight a request, pass what one launch holds.  Every request is looked at,
    empty ones and those that two runs share among them."""
    S, P = (1 << 21) + 5, 256
    lens, N = (0, -3, 1, 63, 64, 65, 128, 200, 255, 256, 300), 13
    pages = randn(N, P, 576, seed=1)
    s = torch.arange(S, device=DEV)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)[s % len(lens)].contiguous()
    table = (s // len(lens) % N).to(torch.int32)[:, None]
    qc, qr = randn(S, 1, 512, seed=2), randn(S, 1, 64, seed=3)
    out, lse = torch.full_like(qc, 3.0), torch.full((1, S), 3.0, device=DEV)
    binding.latent_decode(qc, qr, pages, table, ln, out=out, lse=lse)
    for i, n in enumerate(lens):
        n = min(max(n, 0), P)
        for page in range(N):
            at = s[i::len(lens)]
            at = at[table[at, 0] == page]
            if n == 0:
                assert not bool(out[at].any()) and bool((lse[0, at] == -math.inf).all())
                continue
            o, l, to, tl = ref.decode(qc[at, 0], qr[at, 0], pages[page, :n])
            assert ref.worst(out[at, 0], o, to) <= 1.0, (n, page)
            assert ref.worst(lse[0, at], l, tl) <= 1.0, (n, page, "lse")


def inputs(T, H, seed):
    kv = randn(T, H, 256, seed=seed + 1)
    return randn(T, H, 192, seed=seed), kv[..., :128], randn(T, 576, seed=seed + 2)[:, 512:], kv[..., 128:]


# both sides of the backward in one launch; one after the other, with many heads, and with long sequences
@pytest.mark.parametrize("lens,H", [((700, 64), 5), ((1023,), 10), ((2049, 65), 1), ((1100,), 110), ((4133, 70), 32),
                                    ((8192,), 32)])
def test_norms_of_errors(lens, H):
    """Results and gradients, head by head in blocks of rows or keys (dkr summed over all heads): a tile left out anywhere
    is far outside, and no number of heads hides it."""
    T = sum(lens)
    q, k, kr, v = inputs(T, H, seed=T)
    cu = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device=DEV)
    dout = randn(T, H, 128, seed=T + 9)
    out, lse = binding.latent_forward(q, k, kr, v, cu)
    dq, dk, dkr, dv = binding.latent_backward(q, k, kr, v, cu, out, lse, dout)
    at = 0
    for n in lens:
        s = slice(at, at + n)
        at += n
        sum_, var_ = 0.0, 0.0
        for h in range(H):
            one = slice(h, h + 1)
            r = ref.Attention(q[s, one], k[s, one], kr[s], v[s, one])
            want, _ = r.gradients(dout[s, one])
            var = r.gradient_spread(dout[s, one])
            sum_, var_ = sum_ + want[2], var_ + var[2]
            pairs = [("out", out, r.out, r.out_spread())]
            pairs += [(name, g, want[i], var[i]) for name, g, i in (("dq", dq, 0), ("dk", dk, 1), ("dv", dv, 3))]
            for name, g, x, t in pairs:
                w = ref.worst_block(g[s, one].transpose(0, 1), x, t)
                assert w <= 1.0, (name, n, h, w)
        # (each head's part has the variance of a rounded result in it, a little more than the sum's own)
        w = ref.worst_block(dkr[s], sum_, var_ + ref.U ** 2 / 3 * sum_ ** 2)
        assert w <= 1.0, ("dkr", n, w)
