"""Latent attention at the edges of what its entry points take: the largest calls.  No GPU."""
from paper_2502_13189_amd import binding
from test_abi import lib  # noqa: F401  (fixture)
from test_latent_abi import Backward, Forward


def test_backward_fits_its_launches(lib):  # noqa: F811
    """Delta takes 16 threads a (token, head), dkr 16 a token, in whole work-groups of 256: 2^32 work items are more than
    a launch holds.  The forward has no such launch."""
    most = (1 << 28) - 16
    need = binding.latent_backward_workspace_bytes
    for T, H in ((most + 1, 1), ((1 << 28) - 1, 1), ((1 << 27) - 1, 2)):
        assert Backward(T=T, H=H).call(lib) == "MOBA_ERR_UNSUPPORTED", (T, H)
        assert need(T, H) == 0, (T, H)
    for T, H in ((most, 1), (most // 2, 2)):
        c = Backward(T=T, H=H)
        c.bytes = 100  # (as far as the workspace's check)
        assert c.call(lib) == "MOBA_ERR_NO_MEMORY", (T, H)
        assert need(T, H) == T * H * (8 + 64 * 4)
    c = Forward(T=(1 << 28) - 1, H=1)
    c.t["lse"].dtype = binding.MOBA_BF16  # (its check comes behind that of the size)
    assert c.call(lib) == "MOBA_ERR_DTYPE"
