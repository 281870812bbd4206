"""The entry points of rotary positions and latent attention refuse invalid arguments with the documented
status before touching the device; the workspace queries' arithmetic; the frequencies; the 64-bit
reference's gradients against differences.  No GPU."""
import ctypes
import math

import pytest
import torch

import latent_ref as ref
from paper_2502_13189_amd import binding
from test_abi import FAKE, desc, lib  # noqa: F401  (lib: fixture)

BF, F32, I32, I64, F64 = (binding.MOBA_BF16, binding.MOBA_F32, binding.MOBA_I32, binding.MOBA_I64,
                          binding.MOBA_F64)


def ref_of(d):
    return None if d is None else ctypes.addressof(d)


class Rot(ctypes.Structure):
    _fields_ = [("freqs", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("cu", ctypes.c_void_p),
                ("start", ctypes.c_void_p), ("amplitude", ctypes.c_float), ("interleaved", ctypes.c_int32)]


class Call:
    """Descriptors by name, far apart in a memory that is never read."""

    def __init__(self, **t):
        self.t = t
        for i, d in enumerate(t.values()):
            d.data = FAKE + (i << 40)

    def ref(self, *names):
        return [ref_of(self.t[n]) for n in names]

    def rot(self):
        g = lambda n: ref_of(self.t.get(n))  # noqa: E731
        self.r = Rot(g("freqs"), g("pos"), g("cu"), g("start"), 1.0, 0)
        return ctypes.addressof(self.r)


class Rope(Call):
    names = ("q", "k", "freqs", "pos", "q_out", "k_out")
    fn = "moba_rope"

    def __init__(self, T=7, Hq=4, Hk=2, D=64, rot=64, dtype=BF):
        super().__init__(q=desc([T, Hq, D], dtype), k=desc([T, Hk, D], dtype), freqs=desc([rot // 2], F64),
                         pos=desc([T], I32), q_out=desc([T, Hq, D], dtype), k_out=desc([T, Hk, D], dtype))

    def call(self, lib):
        return binding.STATUS[getattr(lib, self.fn)(*self.ref("q", "k"), self.rot(), *self.ref("q_out", "k_out"), None)]


class RopeBack(Rope):
    fn = "moba_rope_backward"


class Forward(Call):
    names = ("q", "k", "kr", "v", "cu", "out", "lse")

    def __init__(self, T=7, H=3, S=2):
        super().__init__(q=desc([T, H, 192]), k=desc([T, H, 128]), kr=desc([T, 64]), v=desc([T, H, 128]),
                         cu=desc([S + 1], I32), out=desc([T, H, 128]), lse=desc([H, T], F32))
        self.scale = 0.1

    def call(self, lib):
        r = self.ref(*self.names)
        return binding.STATUS[lib.moba_latent_forward(*r[:5], self.scale, *r[5:], None)]


class Backward(Call):
    names = ("q", "k", "kr", "v", "cu", "out", "lse", "dout", "dq", "dk", "dkr", "dv")

    def __init__(self, T=7, H=3, S=2):
        super().__init__(q=desc([T, H, 192]), k=desc([T, H, 128]), kr=desc([T, 64]), v=desc([T, H, 128]),
                         cu=desc([S + 1], I32), out=desc([T, H, 128]), lse=desc([H, T], F32),
                         dout=desc([T, H, 128]), dq=desc([T, H, 192]), dk=desc([T, H, 128]), dkr=desc([T, 64]),
                         dv=desc([T, H, 128]))
        self.scale, self.ws, self.bytes = 0.1, FAKE, 1 << 50

    def call(self, lib):
        r = self.ref(*self.names)
        return binding.STATUS[lib.moba_latent_backward(*r[:5], self.scale, *r[5:], self.ws, self.bytes, None)]


class Write(Call):
    names = ("c", "kr", "slots", "pages", "freqs", "pos")

    def __init__(self, T=7, N=5, P=64):
        super().__init__(c=desc([T, 512]), kr=desc([T, 64]), slots=desc([T], I64), pages=desc([N, P, 576]),
                         freqs=desc([32], F64), pos=desc([T], I64))
        self.turn = True

    def call(self, lib):
        r = self.ref("c", "kr", "slots", "pages")
        return binding.STATUS[lib.moba_latent_write(*r[:3], self.rot() if self.turn else None, r[3], None)]


class Decode(Call):
    names = ("qc", "qr", "pages", "table", "lens", "out", "lse")

    def __init__(self, S=3, H=20, N=9, P=64, W=4):
        super().__init__(qc=desc([S, H, 512]), qr=desc([S, H, 64]), pages=desc([N, P, 576]),
                         table=desc([S, W], I32), lens=desc([S], I32), out=desc([S, H, 512]), lse=desc([H, S], F32))
        self.scale, self.ws, self.bytes = 0.1, FAKE, 1 << 50

    def call(self, lib):
        r = self.ref(*self.names)
        return binding.STATUS[lib.moba_latent_decode(*r[:5], self.scale, *r[5:], self.ws, self.bytes, None)]


ALL = [Rope, RopeBack, Forward, Backward, Write, Decode]


def test_missing(lib):
    for make in ALL:
        for n in make.names:
            c = make()
            c.t[n].data = None
            assert c.call(lib) == "MOBA_ERR_NULL", (make, n)
            c = make()
            c.t[n] = None
            assert c.call(lib) == "MOBA_ERR_NULL", (make, n)
    for make in (Backward, Decode):
        c = make()
        c.ws = None
        assert c.call(lib) == "MOBA_ERR_NULL"


def test_dtypes(lib):
    for make in ALL:
        for n in make.names:
            c = make()
            c.t[n].dtype = binding.MOBA_F8E4M3
            assert c.call(lib) == "MOBA_ERR_DTYPE", (make, n)
    for make in (Forward, Backward, Decode, Write):  # bf16 only
        c = make()
        c.t[make.names[0]].dtype = F32
        assert c.call(lib) == "MOBA_ERR_DTYPE", make
    for n in ("k", "q_out", "k_out"):
        c = Rope()
        c.t[n].dtype = F32  # not as q
        assert c.call(lib) == "MOBA_ERR_DTYPE", n


def test_shapes(lib):
    for make in ALL:
        for n in make.names:
            if n in ("cu", "pages", "freqs") or (make is Decode and n == "table"):
                continue  # (any number of them; their own checks below)
            c = make()
            c.t[n].shape[0] += 1
            assert c.call(lib) == "MOBA_ERR_SHAPE", (make, n)
            c = make()
            c.t[n].ndim -= 1 if c.t[n].ndim > 1 else -1
            assert c.call(lib) == "MOBA_ERR_SHAPE", (make, n)
    for make, n in ((Forward, "v"), (Forward, "out"), (Backward, "dout"), (Backward, "dv"), (Rope, "q_out"),
                    (Rope, "k_out"), (Decode, "qr"), (Decode, "out")):
        c = make()
        d = c.t[n]
        c.t[n] = desc([d.shape[0], d.shape[1] + 1, d.shape[2]], data=d.data)
        assert c.call(lib) == "MOBA_ERR_SHAPE", (make, n)
    for make, n in ((Forward, "q"), (Forward, "kr"), (Backward, "dq"), (Backward, "dkr"), (Write, "c"), (Write, "pages"),
                    (Decode, "qc"), (Decode, "qr"), (Decode, "pages")):
        c = make()
        d = c.t[n]
        d.shape[d.ndim - 1] += 8
        assert c.call(lib) == "MOBA_ERR_UNSUPPORTED", (make, n)
    c = Rope()
    c.t["freqs"].shape[0] = 33  # more pairs than a head has
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    c = Write()
    c.t["freqs"].shape[0] = 31
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    c = Decode()
    c.t["table"].shape[0] = 4
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    for P in (0, 32, 100, 320):
        assert Decode(P=P).call(lib) in ("MOBA_ERR_UNSUPPORTED", "MOBA_ERR_NULL")
        assert Write(P=P).call(lib) in ("MOBA_ERR_UNSUPPORTED", "MOBA_ERR_NULL")


def test_positions(lib):
    c = Rope()  # positions and sequences
    c.t["cu"] = desc([3], I32)
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    for n, dtype in (("cu", I64), ("start", I64)):
        c = Rope()
        c.t["pos"] = None
        c.t["cu"], c.t["start"] = desc([3], I32), desc([2], I32)
        c.t[n].dtype = dtype
        assert c.call(lib) == "MOBA_ERR_DTYPE", n
    c = Rope()
    c.t["pos"] = None
    c.t["cu"], c.t["start"] = desc([3], I32), desc([3], I32)
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    c.t["cu"], c.t["start"] = desc([0], I32), None
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    c = Rope()
    c.t["pos"].stride[0] = 2
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    c = Rope()
    c.t["freqs"].stride[0] = 2
    assert c.call(lib) == "MOBA_ERR_LAYOUT"


def test_layouts(lib):
    for make in ALL:
        for n in make.names:
            d = make().t[n]
            if d.ndim < 2 or n in ("lse", "table"):
                continue
            c = make()
            c.t[n].stride[d.ndim - 1] = 2
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (make, n)
            c = make()
            c.t[n].stride[0] = -8
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (make, n)
            if make in (Rope, RopeBack):
                continue  # (any alignment of an element)
            c = make()
            c.t[n].data += 8
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (make, n)
            c = make()
            c.t[n].stride[0] += 4
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (make, n)
    c = Rope()
    c.t["q"].data += 1
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    for make in (Backward, Decode):
        c = make()
        c.ws += 8
        assert c.call(lib) == "MOBA_ERR_LAYOUT"
    c = Decode()
    c.t["table"].stride[0] = 3
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    for n in ("out", "q_out"):  # rows that lie on each other
        c = Forward() if n == "out" else Rope()
        c.t[n].stride[1] = 64 if n == "out" else 32
        assert c.call(lib) == "MOBA_ERR_LAYOUT", n


def test_overlap(lib):
    """Outputs on inputs, or on each other; views of one buffer whose rows lie apart are no overlap: they get as
    far as the scale's check (a non-positive one) or the piece count's."""
    for make, out, on in ((Forward, "out", "q"), (Forward, "out", "v"), (Backward, "dq", "q"), (Backward, "dk", "dv"),
                          (Backward, "dkr", "kr"), (Backward, "dv", "dout"), (Decode, "out", "qc"),
                          (Rope, "q_out", "k"), (Rope, "k_out", "q"), (Rope, "q_out", "k_out")):
        for shift in (0, 16, -16):
            c = make()
            c.t[out].data = c.t[on].data + shift
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (make, out, on, shift)
    for shift in (2, 128, -128):  # in place, but shifted
        c = Rope()
        c.t["q_out"].data = c.t["q"].data + shift
        assert c.call(lib) == "MOBA_ERR_LAYOUT", shift
    c = Rope()  # the same memory with other strides
    c.t["q_out"].data = c.t["q"].data
    c.t["q_out"].stride[0] += 64
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    # k and v, and their gradients, as views of one [T, H, 256]; the output in a buffer of heads with q
    c = Backward()
    for a, b in (("k", "v"), ("dk", "dv")):
        for n in (a, b):
            c.t[n].stride[0], c.t[n].stride[1] = 3 * 256, 256
        c.t[b].data = c.t[a].data + 256
    c.scale = 0.0
    assert c.call(lib) == "MOBA_ERR_UNSUPPORTED"
    c.t["dv"].data = c.t["dk"].data + 240
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    c = Forward()
    for n, d in (("q", 192), ("out", 128)):
        c.t[n].stride[0], c.t[n].stride[1] = 3 * 320, 320
    c.t["out"].data = c.t["q"].data + 2 * 192
    c.scale = 0.0
    assert c.call(lib) == "MOBA_ERR_UNSUPPORTED"
    c.t["out"].data = c.t["q"].data + 2 * 184
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    # heads outermost
    c = Forward()
    for n, d in (("q", 192), ("out", 128)):
        c.t[n].stride[0], c.t[n].stride[1] = 320, 7 * 320
    c.t["out"].data = c.t["q"].data + 2 * 192
    c.scale = 0.0
    assert c.call(lib) == "MOBA_ERR_UNSUPPORTED"
    c.t["out"].data = c.t["q"].data + 2 * (6 * 320 + 184)
    assert c.call(lib) == "MOBA_ERR_LAYOUT"


def test_overlap_of_the_pool(lib):
    """A write from the pool into itself (its work-groups read and write in any order), a result on the pool; rows that
    lie between the pages of a wider pool are no overlap: such a call gets as far as the next check."""
    for n, at in (("c", 0), ("c", 2 * 5 * 64 * 576 - 1024), ("kr", 2 * 576 * 64 + 1024)):
        c = Write()
        c.t[n].data, c.t[n].stride[0] = c.t["pages"].data + at, 576
        assert c.call(lib) == "MOBA_ERR_LAYOUT", n
        c.turn = False
        assert c.call(lib) == "MOBA_ERR_LAYOUT", n
    c = Write()  # pages of layer 1 of two, tokens in layer 0's page 2
    c.t["pages"].stride[0] = 2 * 64 * 576
    c.t["c"].data, c.t["c"].stride[0] = c.t["pages"].data + 2 * (3 * 64 * 576), 576
    c.t["freqs"].shape[0] = 31
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    c.t["c"].data += 2 * 58 * 576  # its last token in layer 1
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    for at in (0, -2 * 512, 2 * 9 * 64 * 576 - 16):
        c = Decode()
        c.t["out"].data = c.t["pages"].data + at
        assert c.call(lib) == "MOBA_ERR_LAYOUT", at
    c = Decode()
    c.t["out"].data = c.t["pages"].data + 2 * 9 * 64 * 576
    c.scale = 0.0
    assert c.call(lib) == "MOBA_ERR_UNSUPPORTED"


def test_limits(lib):
    for bad in (0.0, -1.0, math.nan, math.inf):
        for make in (Forward, Backward, Decode):
            c = make()
            c.scale = bad
            assert c.call(lib) == "MOBA_ERR_UNSUPPORTED", (make, bad)
    assert Rope(D=1, rot=2).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Rope(D=4098, rot=2).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Forward(T=1 << 21, H=128).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Backward(T=1 << 28, H=1).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Forward(T=10, H=100, S=100000).call(lib) == "MOBA_ERR_UNSUPPORTED"
    c = Forward()
    c.t["k"].stride[0] = 1 << 24
    assert c.call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Decode(H=4097).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Decode(S=1 << 17, H=128, W=1).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Decode(S=1 << 15, H=1, W=1 << 15).call(lib) == "MOBA_ERR_UNSUPPORTED"
    for make in (Backward, Decode):
        c = make()
        c.bytes = 100
        assert c.call(lib) == "MOBA_ERR_NO_MEMORY"


def test_nothing_to_do(lib):
    """No tokens, sequences or requests: no launch, so no device is needed."""
    assert Rope(T=0).call(lib) == "MOBA_OK"
    assert Forward(T=0).call(lib) == "MOBA_OK" and Forward(S=0).call(lib) == "MOBA_OK"
    assert Backward(T=0).call(lib) == "MOBA_OK" and Backward(S=0).call(lib) == "MOBA_OK"
    assert Write(T=0).call(lib) == "MOBA_OK"
    assert Decode(S=0).call(lib) == "MOBA_OK"
    c = Rope(T=0)
    for n in ("q", "k", "pos", "q_out", "k_out"):  # (empty tensors have no memory)
        c.t[n].data = None
    assert c.call(lib) == "MOBA_OK"


def test_workspaces():
    need = binding.latent_decode_workspace_bytes
    for bad in ((0, 4, 8, 64), (-1, 4, 8, 64), (3, 0, 8, 64), (3, 4, 0, 64), (3, 4, 4097, 64), (3, 4, 8, 32),
                (3, 4, 8, 2 ** 40), (2 ** 40, 4, 8, 64), (1 << 15, 1 << 15, 1, 64)):
        assert need(*bad) == 0, bad
    # two partials of a group's heads (512 sums, max and sum) a share, at most as many as steps; the requests'
    # first steps
    pad = lambda n: (n + 15) // 16 * 16  # noqa: E731
    assert need(3, 4, 8, 64) == 12 * 2 * 16 * (512 * 4 + 8) + pad(4 * 4)
    assert need(1, 1 << 14, 128, 64) == 128 * 2 * 2 * 64 * (512 * 4 + 8) + pad(4 * 2)
    back = binding.latent_backward_workspace_bytes
    assert back(0, 3) == back(5, 0) == back(1 << 28, 1) == back(2 ** 40, 1) == 0
    assert back(100, 3) == 300 * (8 + 64 * 4)


def test_binding_checks():
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16)
    r = binding.rotation(64, device="cpu")
    with pytest.raises(ValueError, match="live on a GPU"):
        binding.rope(x, None, r, pos=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="page_size"):
        binding.latent_cache_new(1, 100, device="cpu")
    assert binding.latent_cache_new(3, 192, device="cpu").shape == (3, 192, 576)


def test_rotation():
    for bad in (dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=8, scaling="other"), dict(rot_dim=8, base=0.0),
                dict(rot_dim=8, factor=0.5), dict(rot_dim=2, scaling="base", factor=2.0),
                dict(rot_dim=8, scaling="parts", factor=2.0),
                dict(rot_dim=8, scaling="parts", factor=2.0, original_length=10, low=3.0, high=3.0)):
        with pytest.raises(ValueError):
            binding.rotation(device="cpu", **bad)
    plain = binding.rotation(64, device="cpu")
    assert plain.freqs.dtype == torch.float64 and plain.amplitude == 1.0 and not plain.interleaved
    want = torch.tensor([10000.0 ** (-i / 32) for i in range(32)], dtype=torch.float64)
    assert torch.equal(plain.freqs, want)
    assert torch.equal(binding.rotation(64, scaling="linear", factor=8, device="cpu").freqs, want / 8)
    wide = binding.rotation(64, scaling="base", factor=8, device="cpu")
    assert float(wide.freqs[0]) == 1.0 and abs(float(wide.freqs[-1] * 8 / want[-1]) - 1) < 1e-12
    parts = binding.rotation(64, scaling="parts", factor=8, original_length=4096, device="cpu")
    turns = 4096 * want / (2 * math.pi)
    assert torch.equal(parts.freqs[turns > 32], want[turns > 32])
    assert torch.equal(parts.freqs[turns < 1], want[turns < 1] * (1 / 8))
    mid = (turns >= 1) & (turns <= 32)
    assert bool(((parts.freqs[mid] < want[mid]) & (parts.freqs[mid] > want[mid] / 8)).all()) and int(mid.sum()) > 3
    assert parts.amplitude == 0.1 * math.log(8) + 1.0


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    n, H = 6, 2
    xs = [torch.randn(s, generator=g, dtype=torch.float64) for s in ((n, H, 192), (n, H, 128), (n, 64), (n, H, 128))]
    dout = torch.randn((n, H, 128), generator=g, dtype=torch.float64)
    want, _ = ref.Attention(*xs).gradients(dout)
    want = [x.transpose(0, 1) if x.dim() == 3 else x for x in want]
    h = 1e-5
    for i in range(4):
        d = torch.randn(xs[i].shape, generator=g, dtype=torch.float64)
        loss = [float((ref.Attention(*(x + (s * d if j == i else 0) for j, x in enumerate(xs))).out.transpose(0, 1) *
                       dout).sum()) for s in (h, -h)]
        got, slope = float((want[i] * d).sum()), (loss[0] - loss[1]) / (2 * h)
        assert abs(got - slope) <= 1e-6 * max(1.0, abs(got)), i  # h^2 and 2^-52 / h, both near 1e-10
