"""The paged cache's entry points refuse invalid arguments with the documented status before
touching the device; the workspace query's arithmetic; the binding's own checks.  No GPU."""
import ctypes

import pytest
import torch

from paper_2502_13189_amd import binding
from test_abi import FAKE, desc, lib  # noqa: F401  (lib: fixture)

F8, BF, F32, I32, I64 = (binding.MOBA_F8E4M3, binding.MOBA_BF16, binding.MOBA_F32, binding.MOBA_I32,
                         binding.MOBA_I64)


def ref(d):
    return None if d is None else ctypes.addressof(d)


class Cache:
    def __init__(self, N=10, H=2, P=128):
        self.t = {"k": desc([N, H, P, 128], F8), "v": desc([N, H, 2 * P, 64], F8),
                  "k_scale": desc([N, H], F32), "v_scale": desc([N, H], F32),
                  "k_sum": desc([N, H, 128], F32)}

    def ptr(self):
        self.c = (ctypes.c_void_p * 5)(*(ref(self.t[n]) for n in ("k", "v", "k_scale", "v_scale", "k_sum")))
        return ctypes.addressof(self.c)


class Plan:
    names = ("add", "lens", "table", "free_pages", "num_free", "lens_out", "num_free_out", "cu_new",
             "slots", "refused")

    def __init__(self, S=3, W=4, N=10, T=5, P=64):
        self.t = dict(add=desc([S], I32), lens=desc([S], I32), table=desc([S, W], I32),
                      free_pages=desc([N], I32), num_free=desc([1], I32), lens_out=desc([S], I32),
                      num_free_out=desc([1], I32), cu_new=desc([S + 1], I32), slots=desc([T], I64),
                      refused=desc([1], I32))
        self.P = P

    def call(self, lib):
        p = [ref(self.t[n]) for n in self.names]
        return binding.STATUS[lib.moba_cache_plan(*p[:5], self.P, *p[5:], None)]


class Write:
    def __init__(self, T=7, H=2, dtype=BF, **cache):
        self.t = dict(k=desc([T, H, 128], dtype), v=desc([T, H, 128], dtype), slots=desc([T], I64))
        self.c = Cache(H=H, **cache)

    def call(self, lib):
        return binding.STATUS[lib.moba_cache_write(ref(self.t["k"]), ref(self.t["v"]), ref(self.t["slots"]),
                                                   self.c.ptr(), None)]


class Decode:
    def __init__(self, S=3, W=40, Hq=8, H=2, P=128, block=256, topk=3):
        self.t = dict(q=desc([S, Hq, 128]), table=desc([S, W], I32), lens=desc([S], I32),
                      out=desc([S, Hq, 128], data=1 << 44), lse=desc([Hq, S], F32))
        self.c = Cache(H=H, P=P)
        self.block, self.topk, self.ws, self.bytes = block, topk, FAKE, 1 << 40

    def call(self, lib):
        t = self.t
        return binding.STATUS[lib.moba_cache_decode(ref(t["q"]), self.c.ptr(), ref(t["table"]), ref(t["lens"]),
                                                    self.block, self.topk, ref(t["out"]), ref(t["lse"]),
                                                    self.ws, self.bytes, None)]


def each_missing(make, names, lib):
    for n in names:
        c = make()
        c.t[n].data = None
        assert c.call(lib) == "MOBA_ERR_NULL", n
        c = make()
        c.t[n] = None
        assert c.call(lib) == "MOBA_ERR_NULL", n


def test_missing(lib):
    each_missing(Plan, Plan.names, lib)
    each_missing(Write, ("k", "v", "slots"), lib)
    each_missing(Decode, ("q", "table", "lens", "out", "lse"), lib)
    for make in (Write, Decode):
        for n in ("k", "v", "k_scale", "v_scale", "k_sum"):
            c = make()
            c.c.t[n].data = None
            assert c.call(lib) == "MOBA_ERR_NULL", n
    d = Decode()
    d.ws = None
    assert d.call(lib) == "MOBA_ERR_NULL"


def test_dtypes(lib):
    for n in Plan.names:
        c = Plan()
        c.t[n].dtype = F32
        assert c.call(lib) == "MOBA_ERR_DTYPE", n
    for n in ("k", "v", "slots"):
        c = Write()
        c.t[n].dtype = I32
        assert c.call(lib) == "MOBA_ERR_DTYPE", n
    c = Write()
    c.t["v"].dtype = F32  # k and v differ
    assert c.call(lib) == "MOBA_ERR_DTYPE"
    for n in ("q", "table", "lens", "out", "lse"):
        c = Decode()
        c.t[n].dtype = I64
        assert c.call(lib) == "MOBA_ERR_DTYPE", n
    c = Decode()
    c.t["q"].dtype = F32
    assert c.call(lib) == "MOBA_ERR_DTYPE"
    for make in (Write, Decode):
        for n in ("k", "v", "k_scale", "v_scale", "k_sum"):
            c = make()
            c.c.t[n].dtype = BF
            assert c.call(lib) == "MOBA_ERR_DTYPE", n


def test_shapes(lib):
    for n in Plan.names:
        if n in ("slots", "free_pages"):  # (any length)
            continue
        c = Plan()
        c.t[n].shape[0] += 1
        assert c.call(lib) == "MOBA_ERR_SHAPE", n
    for n in ("k", "v", "slots"):
        c = Write()
        c.t[n].shape[0] += 1
        assert c.call(lib) == "MOBA_ERR_SHAPE", n
    c = Write()
    c.c = Cache(H=3)
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    for n in ("q", "table", "lens", "out", "lse"):
        c = Decode()
        c.t[n].shape[0] += 1
        assert c.call(lib) == "MOBA_ERR_SHAPE", n
    c = Decode()
    c.t["table"].shape[1] = 0
    c.t["table"].data = FAKE
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    c = Decode(Hq=9)
    assert c.call(lib) == "MOBA_ERR_SHAPE"
    for make in (Write, Decode):
        for n in ("v", "k_scale", "v_scale", "k_sum"):
            c = make()
            c.c.t[n].shape[0] += 1
            assert c.call(lib) == "MOBA_ERR_SHAPE", n


def test_layouts(lib):
    for n in ("add", "lens", "cu_new", "slots", "free_pages"):
        c = Plan()
        c.t[n].stride[0] = 2
        assert c.call(lib) == "MOBA_ERR_LAYOUT", n
    c = Plan()
    c.t["table"].stride[1] = 2
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    c = Plan()
    c.t["table"].stride[0] = 3  # rows overlap
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    c = Write()
    c.t["k"].data = FAKE + 2
    assert c.call(lib) == "MOBA_ERR_LAYOUT"
    for make in (Write, Decode):
        for n, i, x in (("k", 0, 128 * 256 + 8), ("v", 1, -16), ("k", 2, 144), ("v", 3, 2), ("k_sum", 1, 256)):
            c = make()
            c.c.t[n].stride[i] = x
            assert c.call(lib) == "MOBA_ERR_LAYOUT", (n, i)
        c = make()
        c.c.t["v"].data = FAKE + 8
        assert c.call(lib) == "MOBA_ERR_LAYOUT"
    d = Decode()
    d.ws = FAKE + 8
    assert d.call(lib) == "MOBA_ERR_LAYOUT"
    for off in (256, 8 * 256, -256):  # out over q, shifted by a head, a row, or back
        d = Decode()
        d.t["q"].data, d.t["out"].data = FAKE * 16, FAKE * 16 + off
        assert d.call(lib) == "MOBA_ERR_LAYOUT"
    d = Decode()  # heads of one wider buffer that do not overlap; the workspace is looked at next
    for n, off in (("q", 0), ("out", 8 * 256)):
        d.t[n].data, d.t[n].stride[0] = FAKE * 16 + off, 16 * 128
    d.bytes = 0
    assert d.call(lib) == "MOBA_ERR_NO_MEMORY"


def test_sizes(lib):
    for P in (32, 96, 320, 0):
        c = Write()
        c.c.t["k"].shape[2] = P
        assert c.call(lib) in ("MOBA_ERR_UNSUPPORTED", "MOBA_ERR_NULL")
    c = Plan()
    c.P = 0
    assert c.call(lib) == "MOBA_ERR_BLOCK_SIZE"
    for P in (32, 100, 512):
        c = Plan()
        c.P = P
        assert c.call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Plan(S=4097).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Plan(S=4096, W=1 << 20).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Plan(N=1 << 31).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Plan(T=1 << 31).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Write(T=1 << 31).call(lib) == "MOBA_ERR_UNSUPPORTED"
    assert Decode(Hq=34).call(lib) == "MOBA_ERR_UNSUPPORTED"  # 17 query heads per kv-head
    assert Decode(topk=-1).call(lib) == "MOBA_ERR_TOPK"
    for block in (0, -128, 64, 129, 192):  # no multiple of the page
        assert Decode(block=block).call(lib) == "MOBA_ERR_BLOCK_SIZE"
    assert Decode(W=4097, block=128).call(lib) == "MOBA_ERR_UNSUPPORTED"  # blocks per row
    assert Decode(S=1 << 22, W=1).call(lib) == "MOBA_ERR_UNSUPPORTED"  # rows
    assert Decode(S=1 << 16, W=1 << 14, topk=0).call(lib) == "MOBA_ERR_UNSUPPORTED"  # steps
    d = Decode()
    d.bytes = binding.cache_decode_workspace_bytes(3, 40, 8, 2, 128, 256, 3) - 1
    assert d.call(lib) == "MOBA_ERR_NO_MEMORY"


def test_nothing_to_do(lib):
    assert Write(T=0).call(lib) == "MOBA_OK"
    assert Decode(S=0).call(lib) == "MOBA_OK"


def test_workspace_bytes(lib):
    f = binding.cache_decode_workspace_bytes
    assert f(0, 40, 8, 2, 128, 256, 3) == 0
    for bad in ((3, 0, 8, 2, 128, 256, 3), (3, 40, 9, 2, 128, 256, 3), (3, 40, 34, 2, 128, 256, 3),
                (3, 40, 8, 2, 100, 256, 3), (3, 40, 8, 2, 128, 200, 3), (3, 40, 8, 2, 128, 256, -1),
                (3, 4097, 8, 2, 128, 128, 3), (-1, 40, 8, 2, 128, 256, 3)):
        assert f(*bad) == 0, bad
    full = f(3, 40, 8, 2, 128, 0, 0)
    assert full > 0
    assert f(3, 40, 8, 2, 128, 256, 20) == full  # top-k covers the row: full attention
    assert f(3, 40, 8, 2, 128, 256, 3) > f(3, 40, 8, 2, 128, 256, 1)
    # does not grow with the lengths that the table can hold, but for the gate's scores
    assert f(1, 1 << 14, 32, 8, 64, 0, 0) == f(1, 1 << 20, 32, 8, 64, 0, 0)


def test_binding_refuses_host_tensors():
    c = binding.cache_new(4, 2, 64, device="cpu")
    i = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.cache_plan(i, i, torch.zeros((2, 3), dtype=torch.int32), i, i[:1], 64, 2)
    with pytest.raises(ValueError):
        binding.cache_write(q, q, torch.zeros(2, dtype=torch.int64), c)
    with pytest.raises(ValueError):
        binding.cache_decode(q, c, torch.zeros((2, 3), dtype=torch.int32), i, 64, 0)
    with pytest.raises(ValueError):
        binding.cache_new(4, 2, 96, device="cpu")
    with pytest.raises(ValueError):
        binding.cache_plan(i, i, torch.zeros((2, 3), dtype=torch.int32), i, i[:1], 64, 2,
                           slots=torch.zeros(3, dtype=torch.int64))
