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
