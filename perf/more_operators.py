"""Rotary positions and latent attention: the calls whose speed matters, as cases to time.

Latent attention keeps one vector of 512 numbers and one rotary key of 64 for each token, which
all heads share.  Prefill and training work on its expanded form, where a head has 128 + 64
numbers for scores (the 64 rotary ones of the key are the shared ones) and 128 for values; decode
works on the absorbed form, where every head scores the 576 cached numbers and sums the 512.

  rope       rotary positions of queries and keys, in both layouts of the pairs, of all or the
             first part of a head, with frequencies as they are or scaled for long contexts
  rope_back  the gradient of that
  prefill    causal latent attention over a packed batch, expanded
  grad       its gradients
  write      new latent vectors and rotary keys, rotated on the way, into the pages of a cache
  decode     one new query per request against its pages, absorbed

With `own` false run() computes them in plain torch operations, with `own` true through
paper_2502_13189_amd.binding.
"""
import math

import torch

own = False

DEV = "cuda:0"
RANK, ROPE, NOPE, VDIM = 512, 64, 128, 128
ROW = RANK + ROPE    # numbers a token has in the cache
QK = NOPE + ROPE     # numbers a head scores in the expanded form
SCALE = 1.0 / math.sqrt(QK)


def _text(xs):
    return ",".join(str(x) for x in xs)


def _rope(name, op, lens, start, hq, hk, dim, rot, pairs=False, dtype="bf16", scaling="none", by="pos"):
    return {"name": name, "op": op, "lens": _text(lens), "start": _text(start), "hq": hq, "hk": hk, "dim": dim,
            "rot": rot, "pairs": pairs, "dtype": dtype, "scaling": scaling, "by": by}


def _attn(name, op, lens, heads):
    return {"name": name, "op": op, "lens": _text(lens), "heads": heads}


def _paged(name, op, lens, page, heads=0, add=(), pairs=False):
    return {"name": name, "op": op, "lens": _text(lens), "page": page, "heads": heads, "add": _text(add), "pairs": pairs}


def _spread(n, lo, hi, salt):
    """n lengths between lo and hi, spread over their logarithm, in no order."""
    return [int(round(lo * (hi / lo) ** (((i * 37 + salt) % n) / max(1, n - 1)))) for i in range(n)]


def listed():
    some = _spread(64, 40, 8000, 5)
    return [
        # a decode step's queries and keys: 64 requests, one token each, at their own positions
        _rope("rope_step", "rope", [1] * 64, some, 32, 8, 128, 128),
        # prompts of a long-context model, packed, with frequencies scaled for it
        _rope("rope_prompts", "rope", (30011, 1, 35000), (0, 517, 900001), 32, 8, 128, 128, scaling="parts", by="seq"),
        # training: gradients of a latent layer's rotary dims (a view of wider heads), interleaved
        _rope("rope_back", "rope_back", (8192, 4099), (0, 0), 40, 1, 64, 64, pairs=True),
        # the smallest prefill: short ragged prompts
        _attn("prefill_small", "prefill", (1, 65, 200, 3, 130), 8),
        # a long prompt
        _attn("prefill_16k", "prefill", (16384,), 32),
        # a training step's packed ragged batch
        _attn("grad_ragged", "grad", (1500, 333, 1, 2049, 700), 10),
        # a training step at full length
        _attn("grad_8k", "grad", (8192,), 32),
        # the decode step's new tokens: one per request, at ragged page offsets
        _paged("write_step", "write", some, 64, add=[1] * 62 + [0, 0], pairs=True),
        # prompts, ragged, and the next piece of a prompt that is partly there
        _paged("write_prompts", "write", (0, 0, 5000, 0, 33), 128, add=(65536, 30000, 4097, 16384, 1000)),
        # the smallest decode call: two short requests and an empty slot of the batch
        _paged("decode_small", "decode", (700, 333, 0), 64, 8),
        # a ragged batch of a chat service
        _paged("decode_ragged", "decode", _spread(48, 100, 30000, 11), 64, 128),
        # the 1M-token cache (the generation of a long-context model)
        _paged("decode_1m", "decode", (1048576,), 128, 128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(c):
    del c["name"]
    return c


def draw(rng):
    op = rng.choice(("rope", "rope", "rope_back", "prefill", "prefill", "grad", "grad", "write", "decode", "decode"))
    if op in ("rope", "rope_back"):
        dim = rng.choice((64, 64, 80, 96, 128, 128, 192, 256, 72, 100))
        rot = rng.choice((dim, dim, dim // 4 * 2, 32, 24))
        hq, hk = rng.choice(((32, 8), (8, 2), (10, 1), (40, 1), (32, 32), (5, 5), (128, 1)))
        n = _log_int(rng, 1, 64)
        tokens = _log_int(rng, n, max(n, 320000000 // (dim * (hq + hk)) // 2))
        lens = [max(1, int(tokens / n * rng.uniform(0.2, 1.0))) for _ in range(n)]
        start = [rng.choice((0, _log_int(rng, 1, 1 << 20))) for _ in lens]
        return _drawn(_rope("", op, lens, start, hq, hk, dim, rot, rng.random() < 0.5,
                            rng.choice(("bf16", "bf16", "f32")), rng.choice(("none", "linear", "base", "parts")),
                            rng.choice(("pos", "seq"))))
    if op in ("prefill", "grad"):
        heads = rng.choice((1, 5, 8, 10, 20, 32, 40, 64, 128))
        n = _log_int(rng, 1, 12)
        top = int(math.sqrt((16384 if op == "prefill" else 8192) ** 2 * 30 / heads / n))
        top = _log_int(rng, 16, min(top, 20000))
        lens = [max(1, int(top * rng.uniform(0.02, 1.0))) for _ in range(n)]
        lens[0] = top
        return _drawn(_attn("", op, lens, heads))
    page = rng.choice((64, 64, 128, 192, 256))
    n = _log_int(rng, 1, 200)
    if op == "write":
        if rng.random() < 0.5:
            lens, add = [_log_int(rng, 1, 8192) for _ in range(n)], [1] * n
        else:
            n = min(n, 16)
            lens = [rng.choice((0, 0, _log_int(rng, 1, 3000))) for _ in range(n)]
            add = [_log_int(rng, 1, 110000 // n) for _ in lens]
        return _drawn(_paged("", "write", lens, page, add=add, pairs=rng.random() < 0.5))
    heads = rng.choice((1, 5, 8, 20, 32, 64, 128, 128))
    top = _log_int(rng, 64, 1000000 // n)
    lens = [max(1, min(top, _log_int(rng, max(1, top // 64), top + 1))) for _ in range(n)]
    if n > 2 and rng.random() < 0.3:
        lens[rng.randrange(n)] = 0
    lens[0] = top
    return _drawn(_paged("", "decode", lens, page, heads))


# ------------------------------------------------------------------- inputs
def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _ceil(a, b):
    return -(-a // b)


#: base, original length, and the factor it is extended by
BASE, ORIGINAL, FACTOR = 10000.0, 32768, 32.0


def _frequencies(rot, scaling):
    """(radians a position [rot / 2] in 64 bits, amplitude): as they are, divided by the
    factor, of a larger base, or between the first two by how often a pair turns over the
    original length."""
    base = BASE * FACTOR ** (rot / (rot - 2)) if scaling == "base" else BASE
    f = [base ** (-2 * i / rot) for i in range(rot // 2)]
    amplitude = 1.0
    if scaling == "linear":
        f = [x / FACTOR for x in f]
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (ORIGINAL * x / (2 * math.pi) - 1.0) / (32.0 - 1.0))) for x in f]
        f = [x * (r + (1 - r) / FACTOR) for x, r in zip(f, keep)]
        amplitude = 0.1 * math.log(FACTOR) + 1.0
    return torch.tensor(f, dtype=torch.float64, device=DEV), amplitude


def _positions(lens, start):
    return torch.cat([torch.arange(b, b + n, device=DEV) for n, b in zip(lens, start)])


def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device=DEV)


def _prepare_rope(case, gen):
    lens, start = _ints(case["lens"]), _ints(case["start"])
    T, dim, rot = sum(lens), case["dim"], case["rot"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    st = {"op": case["op"], "pairs": case["pairs"], "rot": rot, "by": case["by"]}
    # an interleaved case's rotary dims are the end of wider heads, as a latent layer has them
    wide = dim + (NOPE if case["pairs"] else 0)
    q = torch.randn((T, case["hq"], wide), generator=gen, device=DEV).to(dt)
    st["q"] = q[:, :, wide - dim:]
    st["k"] = torch.randn((T, case["hk"], dim), generator=gen, device=DEV).to(dt)
    st["freqs"], st["amplitude"] = _frequencies(rot, case["scaling"])
    st["pos"] = _positions(lens, start).to(torch.int32)
    st["cu"] = _cu(lens)
    st["start"] = torch.tensor(start, dtype=torch.int32, device=DEV)
    return st


def _prepare_attn(case, gen):
    lens, H = _ints(case["lens"]), case["heads"]
    T = sum(lens)
    bf = torch.bfloat16
    st = {"op": case["op"], "longest": max(lens), "cu": _cu(lens)}
    st["q"] = torch.randn((T, H, QK), generator=gen, device=DEV).to(bf)
    # keys and values of a head stand together, as one projection of the latent vector gives them
    kv = torch.randn((T, H, NOPE + VDIM), generator=gen, device=DEV).to(bf)
    st["k"], st["v"] = kv[:, :, :NOPE], kv[:, :, NOPE:]
    # and the rotary key behind the latent vector
    st["kr"] = torch.randn((T, ROW), generator=gen, device=DEV).to(bf)[:, RANK:]
    if case["op"] == "grad":
        fwd = _plain_prefill(st)
        st["out"], st["lse"] = fwd["out"], fwd["lse"]
        st["dout"] = torch.randn((T, H, VDIM), generator=gen, device=DEV).to(bf)
    return st


def _prepare_paged(case, gen):
    P, lens, add = case["page"], _ints(case["lens"]), _ints(case["add"])
    bf = torch.bfloat16
    after = [x + a for x, a in zip(lens, add)] if add else lens
    held = [_ceil(x, P) for x in after]
    n = sum(held) + max(4, sum(held) // 8)
    ids = torch.randperm(n, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros((len(lens), max(1, max(held))), dtype=torch.int32, device=DEV)
    used = 0
    for s, m in enumerate(held):
        table[s, :m] = ids[used:used + m]
        used += m
    st = {"op": case["op"], "pairs": case["pairs"], "page": P, "table": table}
    st["pages"] = torch.empty((n, P, ROW), dtype=bf, device=DEV)
    for i in range(0, n, 1024):  # whole pages hold numbers: what a request does not have is not read
        st["pages"][i:i + 1024] = torch.randn((min(1024, n - i), P, ROW), generator=gen, device=DEV)
    if case["op"] == "write":
        pos = _positions(add, lens)
        who = torch.repeat_interleave(torch.arange(len(add), device=DEV), torch.tensor(add, device=DEV))
        slots = table[who, pos // P].long() * P + pos % P
        # a padded batch: the last rows of the call are no tokens
        st["slots"] = torch.cat([slots, torch.full((3,), -1, device=DEV, dtype=torch.int64)])
        st["pos"] = torch.cat([pos, pos.new_zeros(3)]).to(torch.int32)
        st["c"] = torch.randn((pos.numel() + 3, RANK), generator=gen, device=DEV).to(bf)
        st["kr"] = torch.randn((pos.numel() + 3, ROPE), generator=gen, device=DEV).to(bf)
        st["freqs"], st["amplitude"] = _frequencies(ROPE, "parts")
        return st
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    st["qc"] = torch.randn((len(lens), case["heads"], RANK), generator=gen, device=DEV).to(bf)
    # the rotary part is a view of the heads' queries
    st["qr"] = torch.randn((len(lens), case["heads"], QK), generator=gen, device=DEV).to(bf)[:, :, NOPE:]
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if case["op"] in ("rope", "rope_back"):
        return _prepare_rope(case, gen)
    if case["op"] in ("prefill", "grad"):
        return _prepare_attn(case, gen)
    return _prepare_paged(case, gen)


# -------------------------------------------------------------- plain forms
def _turn(x, pos, freqs, amplitude, pairs, sign):
    """x [T, H, D] with its first 2 * len(freqs) dims rotated by sign * pos * freqs."""
    n = freqs.numel()
    angle = pos.double()[:, None] * freqs
    c = (angle.cos() * amplitude).float()[:, None]
    s = (angle.sin() * (amplitude * sign)).float()[:, None]
    y = x.float()
    a, b = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if pairs else (y[..., :n], y[..., n:2 * n])
    a, b = a * c - b * s, a * s + b * c
    y = y.clone()
    if pairs:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = a, b
    else:
        y[..., :n], y[..., n:2 * n] = a, b
    return y.to(x.dtype)


def _plain_rope(st):
    sign = -1.0 if st["op"] == "rope_back" else 1.0
    return {n: _turn(st[n], st["pos"], st["freqs"], st["amplitude"], st["pairs"], sign) for n in ("q", "k")}


def _rows(st):
    """Token of every place [S, longest] of the padded batch, and whether it is one."""
    cu = st["cu"].long()
    at = torch.arange(st["longest"], device=DEV)
    ok = at < (cu[1:] - cu[:-1])[:, None]
    return torch.where(ok, cu[:-1, None] + at, 0), ok


def _chunks(S, H, n):
    """(sequences, heads) whose scores are taken at once."""
    heads = max(1, min(H, (1 << 31) // (n * n)))
    seqs = max(1, min(S, (1 << 31) // (n * n * heads)))
    return [(slice(s, s + seqs), slice(h, h + heads)) for s in range(0, S, seqs) for h in range(0, H, heads)]


def _padded(x, row, heads):
    """x [T, H, D] -> [S, heads, longest, D] in 32 bits."""
    return x[row][:, :, heads].transpose(1, 2).float().contiguous()


def _scores(st, row, heads):
    """Scaled scores [S, heads, n, n], the future masked, and the queries and keys in 32 bits."""
    q = _padded(st["q"], row, heads)
    k = _padded(st["k"], row, heads)
    k = torch.cat([k, _padded(st["kr"][:, None], row, slice(0, 1)).expand(-1, k.shape[1], -1, -1)], 3)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(SCALE)
    n = torch.arange(row.shape[1], device=DEV)
    return z.masked_fill_(n > n[:, None], -math.inf), q, k


def _plain_prefill(st):
    T, H = st["q"].shape[:2]
    out = torch.empty((T, H, VDIM), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((H, T), device=DEV)
    row, ok = _rows(st)
    for s, h in _chunks(row.shape[0], H, row.shape[1]):
        z, _, _ = _scores(st, row[s], h)
        m = z.amax(3, keepdim=True)
        p = z.sub_(m).exp_()
        l = p.sum(3, keepdim=True)
        o = torch.matmul(p, _padded(st["v"], row[s], h)) / l
        r = row[s][ok[s]]
        out[r, h] = o.transpose(1, 2)[ok[s]].to(torch.bfloat16)
        lse[h, r] = (l.log() + m)[..., 0].transpose(1, 2)[ok[s]].t()
    return {"out": out, "lse": lse}


def _plain_grad(st):
    T, H = st["q"].shape[:2]
    bf = torch.bfloat16
    dq = torch.empty((T, H, QK), dtype=bf, device=DEV)
    dk = torch.empty((T, H, NOPE), dtype=bf, device=DEV)
    dv = torch.empty((T, H, VDIM), dtype=bf, device=DEV)
    dkr = torch.zeros((T, ROPE), device=DEV)
    row, ok = _rows(st)
    for s, h in _chunks(row.shape[0], H, row.shape[1]):
        z, q, k = _scores(st, row[s], h)
        p = z.sub_(st["lse"][h][:, row[s]].transpose(0, 1)[..., None]).exp_()
        p *= ok[s][:, None, :, None]  # places that are no tokens have no gradient
        do = _padded(st["dout"], row[s], h)
        r = row[s][ok[s]]
        dv[r, h] = torch.matmul(p.transpose(2, 3).contiguous(), do).transpose(1, 2)[ok[s]].to(bf)
        dp = torch.matmul(do, _padded(st["v"], row[s], h).transpose(2, 3).contiguous())
        ds = dp.sub_((p * dp).sum(3, keepdim=True)).mul_(p).mul_(SCALE)
        dq[r, h] = torch.matmul(ds, k).transpose(1, 2)[ok[s]].to(bf)
        g = torch.matmul(ds.transpose(2, 3).contiguous(), q).transpose(1, 2)[ok[s]]
        dk[r, h] = g[..., :NOPE].to(bf)
        dkr[r] += g[..., NOPE:].sum(1)
    return {"dq": dq, "dk": dk, "dkr": dkr.to(bf), "dv": dv}


def _plain_write(st):
    slots = st["slots"]
    ok = slots >= 0
    kr = _turn(st["kr"][:, None], st["pos"], st["freqs"], st["amplitude"], st["pairs"], 1.0)[:, 0]
    rows = st["pages"].view(-1, ROW)
    # rows that are no tokens repeat the first one, which is
    row = torch.where(ok, torch.arange(slots.numel(), device=DEV), 0)
    rows[slots[row]] = torch.cat([st["c"], kr], 1)[row]
    return {"pages": st["pages"]}


def _plain_decode(st):
    S, H = st["qc"].shape[:2]
    P, idx = st["page"], st["table"].long()
    n = idx.shape[1] * P
    out = torch.empty((S, H, RANK), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((H, S), device=DEV)
    pos = torch.arange(n, device=DEV)
    step = max(1, (1 << 20) // n)  # requests at a time
    for s in range(0, S, step):
        e = min(S, s + step)
        u = st["pages"][idx[s:e]].view(e - s, n, ROW).float()
        q = torch.cat([st["qc"][s:e], st["qr"][s:e]], 2).float()
        use = (pos < st["lens"][s:e, None])[:, None]
        z = torch.matmul(q, u.transpose(1, 2)) * SCALE
        z = torch.where(use, z, -math.inf)
        m = z.amax(2, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)
        p = z.sub_(m).exp_()
        l = p.sum(2, keepdim=True)
        o = torch.matmul(p, torch.where(use.transpose(1, 2), u[..., :RANK], 0.0)) / torch.where(l > 0, l, 1.0)
        out[s:e] = o.to(torch.bfloat16)
        lse[:, s:e] = (l.log() + m)[..., 0].t()
    return {"out": out, "lse": lse}


_PLAIN = {"rope": _plain_rope, "rope_back": _plain_rope, "prefill": _plain_prefill, "grad": _plain_grad,
          "write": _plain_write, "decode": _plain_decode}


def run(state):
    op = state["op"]
    if not own:
        return _PLAIN[op](state)
    from paper_2502_13189_amd import binding
    if op in ("rope", "rope_back"):
        rot = binding.Rotation(state["freqs"], state["amplitude"], state["pairs"])
        at = {"pos": state["pos"]} if state["by"] == "pos" else {"cu_seqlens": state["cu"], "start": state["start"]}
        f = binding.rope if op == "rope" else binding.rope_backward
        q, k = f(state["q"], state["k"], rot, **at)
        return {"q": q, "k": k}
    if op == "prefill":
        out, lse = binding.latent_forward(state["q"], state["k"], state["kr"], state["v"], state["cu"])
        return {"out": out, "lse": lse}
    if op == "grad":
        dq, dk, dkr, dv = binding.latent_backward(state["q"], state["k"], state["kr"], state["v"], state["cu"],
                                                  state["out"], state["lse"], state["dout"])
        return {"dq": dq, "dk": dk, "dkr": dkr, "dv": dv}
    if op == "write":
        rot = binding.Rotation(state["freqs"], state["amplitude"], state["pairs"])
        binding.latent_write(state["c"], state["kr"], state["slots"], state["pages"], rot, pos=state["pos"])
        return {"pages": state["pages"]}
    out, lse = binding.latent_decode(state["qc"], state["qr"], state["pages"], state["table"], state["lens"])
    return {"out": out, "lse": lse}


def work(case):
    op, lens = case["op"], _ints(case["lens"])
    if op in ("rope", "rope_back"):
        T, H, el = sum(lens), case["hq"] + case["hk"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * T * H * case["dim"] * el + 4 * T, "flops": 3 * T * H * case["rot"]}
    if op in ("prefill", "grad"):
        T, H = sum(lens), case["heads"]
        scored = H * sum(n * (n + 1) // 2 for n in lens)
        fwd = T * H * (QK + NOPE + 2 * VDIM) * 2 + T * ROPE * 2 + 4 * T * H
        if op == "prefill":
            return {"bytes": fwd, "flops": 2 * scored * (QK + VDIM)}
        return {"bytes": fwd + T * H * (QK + NOPE + 2 * VDIM) * 2 + T * ROPE * 2,
                "flops": 2 * scored * (3 * QK + 2 * VDIM)}
    if op == "write":
        T = sum(_ints(case["add"]))
        return {"bytes": T * (2 * ROW * 2 + 12), "flops": 3 * T * ROPE}
    S, H = len(lens), case["heads"]
    return {"bytes": sum(lens) * ROW * 2 + S * H * (ROW + RANK) * 2 + 4 * S * H,
            "flops": 2 * H * sum(lens) * (ROW + RANK)}


# ------------------------------------------------------------------ 64 bits
def _exact_turn(x, case, st, sign):
    """Rotation as a product with exp(i angle)."""
    T = x.shape[0]
    n = st["freqs"].numel()
    y = x.double().clone()
    z = y[..., :2 * n].reshape(T, -1, n, 2) if case["pairs"] else y[..., :2 * n].reshape(T, -1, 2, n).transpose(2, 3)
    # the angle in turns, whole ones taken off
    turns = st["pos"].double()[:, None] * (st["freqs"] / (2 * math.pi))
    angle = (turns - turns.round()) * (2 * math.pi) * sign
    w = torch.polar(torch.full_like(angle, st["amplitude"]), angle)[:, None]
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * w)
    y[..., :2 * n] = (z if case["pairs"] else z.transpose(2, 3)).reshape(T, -1, 2 * n)
    return y


def _exact_attn(case, st):
    H = case["heads"]
    z64 = dict(dtype=torch.float64, device=DEV)
    T = st["q"].shape[0]
    out, lse = torch.zeros((T, H, VDIM), **z64), torch.zeros((H, T), **z64)
    dq, dk, dkr, dv = (torch.zeros(s, **z64) for s in ((T, H, QK), (T, H, NOPE), (T, ROPE), (T, H, VDIM)))
    at = 0
    for n in _ints(case["lens"]):
        r = slice(at, at + n)
        at += n
        future = torch.ones((n, n), dtype=torch.bool, device=DEV).triu_(1)
        kr = st["kr"][r].double()
        for h in range(H):
            q, k, v = st["q"][r, h].double(), st["k"][r, h].double(), st["v"][r, h].double()
            z = (q[:, :NOPE] @ k.t() + q[:, NOPE:] @ kr.t()) / math.sqrt(QK)
            z.masked_fill_(future, -math.inf)
            lse[h, r] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            o = p @ v
            out[r, h] = o
            if case["op"] == "grad":
                g = st["dout"][r, h].double()
                dv[r, h] = p.t() @ g
                # softmax's gradient: p (g - <g, p>), where <dp, p> is <dout, out>
                ds = p * (g @ v.t() - (g * o).sum(1, keepdim=True)) / math.sqrt(QK)
                dq[r, h, :NOPE] = ds @ k
                dq[r, h, NOPE:] = ds @ kr
                dk[r, h] = ds.t() @ q[:, :NOPE]
                dkr[r] += ds.t() @ q[:, NOPE:]
    return {"out": out, "lse": lse} if case["op"] == "prefill" else {"dq": dq, "dk": dk, "dkr": dkr, "dv": dv}


def _exact_write(case, st):
    pages = st["pages"].double()
    kr = _exact_turn(st["kr"][:, None], case, st, 1)[:, 0]
    for t0 in range(0, st["slots"].numel(), 4096):
        t = t0 + torch.nonzero(st["slots"][t0:t0 + 4096] >= 0)[:, 0]
        page = torch.div(st["slots"][t], case["page"], rounding_mode="floor")
        off = st["slots"][t] - page * case["page"]
        pages[page, off, :RANK] = st["c"][t].double()
        pages[page, off, RANK:] = kr[t]
    return {"pages": pages}


def _exact_decode(case, st):
    S, H = st["qc"].shape[:2]
    out = torch.zeros((S, H, RANK), dtype=torch.float64, device=DEV)
    lse = torch.full((H, S), -math.inf, dtype=torch.float64, device=DEV)
    for s, n in enumerate(_ints(case["lens"])):
        if not n:
            continue
        u = st["pages"][st["table"][s, :_ceil(n, case["page"])].long()].reshape(-1, ROW)[:n].double()
        z = (st["qc"][s].double() @ u[:, :RANK].t() + st["qr"][s].double() @ u[:, RANK:].t()) / math.sqrt(QK)
        lse[:, s] = torch.logsumexp(z, 1)
        out[s] = torch.softmax(z, 1) @ u[:, :RANK]
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("rope", "rope_back"):
        sign = 1 if case["op"] == "rope" else -1
        return {n: _exact_turn(st[n], case, st, sign) for n in ("q", "k")}
    if case["op"] in ("prefill", "grad"):
        return _exact_attn(case, st)
    return (_exact_write if case["op"] == "write" else _exact_decode)(case, st)
