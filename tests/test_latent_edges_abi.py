"""Latent attention and rotary positions at the edges of what their entry points take: the largest calls, tensors that
share memory.  No GPU."""
import pytest

from paper_2502_13189_amd import binding
from test_abi import FAKE, desc, lib  # noqa: F401  (lib: fixture)
from test_latent_abi import Backward, Decode, Forward, Rope, Write


def size(d):
    """Bytes of a contiguous descriptor."""
    n = {binding.MOBA_BF16: 2, binding.MOBA_F32: 4, binding.MOBA_I32: 4, binding.MOBA_I64: 8, binding.MOBA_F64: 8}[d.dtype]
    for i in range(d.ndim):
        n *= d.shape[i]
    return n


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


def up(n):
    return -(-n // 16) * 16


def next_check(c):
    """A call that gets past the overlap of its tensors is refused by the scale or for the workspace's size."""
    if isinstance(c, Forward):
        c.scale = 0.0
    else:
        c.bytes = 100


# what a call writes beside its bf16 rows, and every tensor that lies beside it
WRITTEN = [(Forward, "lse"), (Decode, "lse"), (Forward, "out"), (Decode, "out"), (Backward, "dq"), (Backward, "dkr")]


@pytest.mark.parametrize("make,written", WRITTEN)
def test_overlap_with_every_other_tensor(lib, make, written):  # noqa: F811
    """On its first and its last 16 bytes; directly before and behind it, they share nothing."""
    for n in make.names:
        if n == written:
            continue
        w, d = size(make().t[written]), size(make().t[n])
        for at, share in ((0, True), (up(d) - 16, True), (16 - up(w), True), (up(d), False), (-up(w), False)):
            c = make()
            c.t[written].data = c.t[n].data + at
            next_check(c)
            apart = "MOBA_ERR_UNSUPPORTED" if make is Forward else "MOBA_ERR_NO_MEMORY"
            assert c.call(lib) == ("MOBA_ERR_LAYOUT" if share else apart), (make, written, n, at)


@pytest.mark.parametrize("make", [Backward, Decode])
def test_overlap_of_the_workspace(lib, make):  # noqa: F811
    """What the call uses of it: bytes behind that may hold anything."""
    if make is Backward:
        need = binding.latent_backward_workspace_bytes(7, 3)
    else:
        need = binding.latent_decode_workspace_bytes(3, 4, 20, 64)
    for n in make.names:
        for at in (0, up(size(make().t[n])) - 16, 16 - need):
            c = make()
            c.t[n].data += 1 << 39  # (the first tensor lies lower than a workspace is large)
            c.ws = c.t[n].data + at
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (n, at)


def test_results_between_the_pages_of_a_wider_pool(lib):  # noqa: F811
    """A page stride wider than a page leaves room that is not the pool's."""
    c = Decode()
    c.t["pages"].stride[0] = 2 * 64 * 576
    c.t["lse"].data = c.t["pages"].data + 2 * 64 * 576
    c.bytes = 100
    assert c.call(lib) == "MOBA_ERR_NO_MEMORY"
    for at in (-16, 2 * 64 * 576 - 16):  # its first bytes or its last ones in a page
        c.t["lse"].data = c.t["pages"].data + 2 * 64 * 576 + at
        assert c.call(lib) == "MOBA_ERR_LAYOUT", at


def test_overlap_with_slots_and_positions(lib):  # noqa: F811
    """The pool of a write, and rotary results, on what says where and how far rows are turned."""
    def seqs(c, S=2):
        c.t["pos"] = None
        c.t["cu"], c.t["start"] = desc([S + 1], binding.MOBA_I32), desc([S], binding.MOBA_I32)
        c.t["cu"].data, c.t["start"].data = FAKE + (20 << 40), FAKE + (21 << 40)
        return c

    for n in ("slots", "freqs", "pos"):
        c = Write()
        c.t["pages"].data = c.t[n].data
        assert c.call(lib) == "MOBA_ERR_LAYOUT", n
    for n in ("cu", "start"):
        c = seqs(Write())
        c.t["pages"].data = c.t[n].data
        assert c.call(lib) == "MOBA_ERR_LAYOUT", n
        for out in ("q_out", "k_out"):
            c = seqs(Rope())
            c.t[out].data = c.t[n].data
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (out, n)
    for n in ("freqs", "pos"):
        for out in ("q_out", "k_out"):
            c = Rope()
            c.t[out].data = c.t[n].data
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (out, n)
