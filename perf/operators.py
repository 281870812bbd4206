"""Serving from a paged 8-bit key/value cache: the calls whose speed matters, as cases to time.

The cache holds pages of `page` tokens.  For each page and kv-head it has the keys as e4m3
[page, 128], the values as e4m3 with the token index innermost [page / 64, 128, 64], one
power-of-two scale each, and the fp32 sum of the page's keys (what the MoBA gate scores).
Three operators work on it:

  plan    the step's block tables and slot maps from the requests' lengths: pages come off
          a free list (those of ended requests go back first), every new token gets its
          slot, page * page_size + offset
  write   new keys and values into their slots, quantised
  decode  one new query per request against its pages, full attention (topk 0) or MoBA

With `own` false run() computes them in plain torch operations, with `own` true through
paper_2502_13189_amd.binding.
"""
import math

import torch

own = False

DEV = "cuda:0"
D = 128
F8 = torch.float8_e4m3fn
E_MIN, E_MAX = -100, 119  # exponents of a scale


def _case(name, op, lens, page, hkv=0, hq=0, add="", block=0, topk=0, dtype="bf16"):
    return {"name": name, "op": op, "lens": lens, "add": add, "page": page, "hkv": hkv, "hq": hq,
            "block": block, "topk": topk, "dtype": dtype}


def _text(xs):
    return ",".join(str(x) for x in xs)


def _spread(n, lo, hi, salt):
    """n lengths between lo and hi, spread over their logarithm, in no order."""
    return [int(round(lo * (hi / lo) ** (((i * 37 + salt) % n) / max(1, n - 1)))) for i in range(n)]


def listed():
    some = _spread(64, 40, 8000, 5)
    return [
        # a decode step of a full batch: 61 requests grow by a token, two end, one slot is empty
        _case("plan_step", "plan", _text(some[:63] + [0]), 64,
              add=_text([-1 if i in (7, 40) else 0 if i == 63 else 1 for i in range(64)])),
        # prompts of 1M tokens in all enter an empty batch
        _case("plan_prompts", "plan", _text([0] * 8), 64,
              add=_text([524288, 131072, 100003, 1, 65536, 131072, 777, 95827])),
        # the same step's keys and values: one token per request, at ragged page offsets
        _case("write_step", "write", _text(some), 64, 8, add=_text([1] * 62 + [0, 0])),
        # prompts, ragged, and the next piece of a prompt that is partly there
        _case("write_prompts", "write", "0,0,5000,0,33", 128, 8,
              add="65536,30000,4097,16384,1000"),
        # fp32 keys and values of two short prompts
        _case("write_f32", "write", "0,0", 64, 2, add="700,333", dtype="f32"),
        # the smallest decode call: two short requests and an empty slot of the batch
        _case("decode_small", "decode", "700,333,0", 64, 2, 8),
        # a ragged batch, full attention
        _case("decode_ragged", "decode", "30011,512,9000,65536,1,4097,16384,2300", 64, 8, 32),
        # many requests of a chat's length, multi-head attention
        _case("decode_many", "decode", _text(_spread(192, 16, 4096, 11)), 128, 32, 32),
        # the 1M-token cache, full attention (the generation of a long-context model)
        _case("decode_1m", "decode", "1048576", 64, 8, 32),
        # a ragged batch, MoBA
        _case("moba_ragged", "decode", "30011,70000,9000,65536,1,12288,131072,2300", 64, 8, 32,
              block=1024, topk=4),
        # the 1M-token cache, MoBA
        _case("moba_1m", "decode", "1048576", 128, 8, 32, block=4096, topk=12),
    ]


#: query heads, kv-heads
_HEADS = [(4, 4), (8, 2), (12, 4), (16, 2), (16, 1), (32, 8), (32, 32)]
_PAGES = (64, 64, 128, 192, 256)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("plan", "write", "decode", "decode", "moba", "moba"))
    page = rng.choice(_PAGES)
    hq, hkv = rng.choice(_HEADS)
    n = _log_int(rng, 1, 256)
    if op == "plan":
        if rng.random() < 0.5:
            lens = [_log_int(rng, 1, 20000) for _ in range(n)]
            add = [rng.choice((1, 1, 1, 1, 1, 1, 1, 1, 0, -1)) for _ in lens]
        else:
            n = min(n, 32)
            lens = [rng.choice((0, _log_int(rng, 1, 9000))) for _ in range(n)]
            add = [_log_int(rng, 1, (1 << 20) // n) for _ in lens]
        return _drawn("plan", lens, page, add=add)
    if op == "write":
        if rng.random() < 0.5:
            lens, add = [_log_int(rng, 1, 8192) for _ in range(n)], [1] * n
        else:
            n = min(n, 16)
            lens = [rng.choice((0, 0, _log_int(rng, 1, 3000))) for _ in range(n)]
            add = [_log_int(rng, 1, 131072 // n) for _ in lens]
        return _drawn("write", lens, page, hkv, add=add, dtype=rng.choice(("bf16", "bf16", "f32")))
    # the padded table has at most 8M (token, kv-head) pairs
    most = min(1 << 20, (1 << 23) // hkv // n)
    top = _log_int(rng, 64, most)
    lens = [max(1, min(top, _log_int(rng, max(1, top // 64), top + 1))) for _ in range(n)]
    if n > 2 and rng.random() < 0.3:
        lens[rng.randrange(n)] = 0
    lens[0] = top
    if op == "decode":
        return _drawn("decode", lens, page, hkv, hq)
    block = page * _log_int(rng, 1, max(1, min(4096, top // 3) // page))
    return _drawn("decode", lens, page, hkv, hq, block=max(block, -(-top // (2048 * page)) * page),
                  topk=rng.choice((2, 3, 4, 4, 8, 12, 16, 32)))


def _drawn(op, lens, page, hkv=0, hq=0, add=(), **more):
    c = _case("", op, _text(lens), page, hkv, hq, _text(add), **more)
    del c["name"]
    return c


# ------------------------------------------------------------------- inputs
def _ints(text):
    return [int(x) for x in text.split(",")]


def _ceil(a, b):
    return -(-a // b)


def _pool(case, lens, gen):
    """(pages in the pool, width of the table, each request's pages): page ids in no order."""
    held = [_ceil(x, case["page"]) for x in lens]
    n = sum(held) + max(4, sum(held) // 8)
    ids = torch.randperm(n, generator=gen, device=DEV).to(torch.int32)
    return n, held, ids


def _to_f8(x):
    return x.to(F8).view(torch.uint8)


def _scale_of(amax):
    """The least power of two 2^e with amax <= 448 * 2^e, e in [E_MIN, E_MAX]; as e."""
    m, e = torch.frexp(amax)
    return (e - 8 - (m <= 0.875).to(e.dtype)).clamp(E_MIN, E_MAX)


def _filled(case, lens, table, n, gen):
    """A pool whose pages hold the requests' keys and values: Gaussian, the keys of a MoBA
    block with an offset of their own, quantised by page and kv-head."""
    P, H = case["page"], case["hkv"]
    kp = torch.zeros((n, H, P, D), dtype=torch.uint8, device=DEV)
    vp = torch.zeros((n, H, P // 64, D, 64), dtype=torch.uint8, device=DEV)
    ks = torch.ones((n, H), device=DEV)
    vs = torch.ones((n, H), device=DEV)
    ksum = torch.zeros((n, H, D), device=DEV)
    B = case["block"] or 2048
    step = max(1, (1 << 27) // (H * P * D))
    for s, L in enumerate(lens):
        for j0 in range(0, _ceil(L, P), step):
            j1 = min(_ceil(L, P), j0 + step)
            at = table[s, j0:j1].long()
            tok = torch.arange(j0 * P, j1 * P, device=DEV)
            off = torch.randn((int(tok[-1]) // B - j0 * P // B + 1, H, D), generator=gen, device=DEV) * 0.5
            for is_k in (True, False):
                x = torch.randn((j1 - j0, P, H, D), generator=gen, device=DEV)
                if is_k:
                    x += off[tok // B - j0 * P // B].view(j1 - j0, P, H, D)
                x *= (tok < L).view(j1 - j0, P, 1, 1)
                e = _scale_of(x.abs().amax((1, 3)))
                b = _to_f8(torch.ldexp(x, -e[:, None, :, None])).permute(0, 2, 1, 3)
                (ks if is_k else vs)[at] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
                if is_k:
                    kp[at] = b
                    ksum[at] = (b.view(F8).double().sum(2) * ks[at].double()[..., None]).float()
                else:
                    vp[at] = b.reshape(j1 - j0, H, P // 64, 64, D).transpose(3, 4)
    return {"k": kp.view(F8), "v": vp.view(F8), "k_scale": ks, "v_scale": vs, "k_sum": ksum}


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, P, lens = case["op"], case["page"], _ints(case["lens"])
    add = _ints(case["add"]) if case["add"] else [0] * len(lens)
    n_new = sum(max(a, 0) for a in add)
    after = [max(x, x + max(a, 0)) for x, a in zip(lens, add)]
    n, held, ids = _pool(case, after, gen)
    S = len(lens)
    width = max(1, max(held))
    table = torch.zeros((S, width), dtype=torch.int32, device=DEV)
    # a plan starts from the pages held before it, the other operators have its result
    have = [_ceil(x, P) for x in lens] if op == "plan" else held
    used = 0
    for s, m in enumerate(have):
        table[s, :m] = ids[used:used + m]
        used += m
    st = {"op": op, "page": P, "table": table}
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if op == "plan":
        st["add"] = torch.tensor(add, dtype=torch.int32, device=DEV)
        st["free"] = ids.roll(-used).contiguous()  # the pages in use stand behind the free ones
        st["num_free"] = torch.tensor([n - used], dtype=torch.int32, device=DEV)
        st["tokens"] = n_new + n_new // 50 + 3  # room for more tokens than come
        return st
    st["cache"] = _filled(case, lens, table, n, gen)
    if op == "write":
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        slots = [torch.arange(x, x + a, device=DEV) for x, a in zip(lens, add)]
        slots = torch.cat([table[s][t // P].long() * P + t % P for s, t in enumerate(slots)])
        # a padded batch: the last rows of the call are no tokens
        st["slots"] = torch.cat([slots, torch.full((3,), -1, device=DEV, dtype=torch.int64)])
        T = st["slots"].numel()
        # a token's size differs from the others', as activations' do
        size = torch.exp(0.5 * torch.randn((T, 1, 1), generator=gen, device=DEV))
        for name in ("k", "v"):
            x = torch.randn((T, case["hkv"], D), generator=gen, device=DEV)
            st[name] = x.mul_(size).to(dt)
        # how many runs of tokens the pages cut the call into
        st["runs"] = sum(_ceil(x + a, P) - x // P for x, a in zip(lens, add) if a)
        return st
    st["q"] = torch.randn((S, case["hq"], D), generator=gen, device=DEV).to(torch.bfloat16)
    st["block"], st["topk"] = case["block"], case["topk"]
    return st


# -------------------------------------------------------------- plain forms
def _plain_plan(st):
    add, lens, P = st["add"].long(), st["lens"].long(), st["page"]
    table, free, T = st["table"], st["free"], st["tokens"]
    S, W = table.shape
    n = free.numel()
    ended = add < 0
    tok = add.clamp(min=0)
    held = (lens + P - 1) // P
    after = torch.where(ended, torch.zeros_like(lens), lens + tok)
    upto = tok.cumsum(0)
    fits = ~ended & ((after + P - 1) // P <= W) & (upto <= T)
    need = torch.where(fits, (after + P - 1) // P - held, 0)
    back = torch.where(ended, held, 0)
    avail = st["num_free"].long() + back.sum()
    granted = fits & ((need == 0) | (need.cumsum(0) <= avail))
    take = torch.where(granted, need, 0)
    # pages of ended requests go back, then pages are taken from the end
    j = torch.arange(W, device=DEV)[None]
    room = torch.cat([free, free[:1]])
    to = st["num_free"].long() + (back.cumsum(0) - back)[:, None] + j
    to = torch.where(j < back[:, None], to, n).clamp(max=n)
    room[to.reshape(-1)] = table.reshape(-1)
    free.copy_(room[:n])
    i = (take.cumsum(0) - take)[:, None] + j - held[:, None]
    mine = (j >= held[:, None]) & (j < (held + take)[:, None])
    page = free[torch.where(mine, avail - 1 - i, 0).clamp(0, n - 1)]
    table.copy_(torch.where(mine, page, table))
    new_lens = torch.where(granted | ended, after, lens)
    cu = torch.cat([torch.zeros_like(upto[:1]), upto]).clamp(max=T)
    t = torch.arange(T, device=DEV)
    s = torch.searchsorted(upto, t, right=True)
    ok = s < S
    s = s.clamp(max=S - 1)
    pos = lens[s] + t - cu[s]
    ok &= granted[s]
    slot = table[s, torch.where(ok, pos // P, 0)].long() * P + pos % P
    return {"cu": cu.int(), "slots": torch.where(ok, slot, -1), "lens": new_lens.int(),
            "num_free": (avail - take.sum()).int(), "table": table, "free": free,
            "refused": (~granted & ~ended).sum().int().view(1)}


def _plain_write(st):
    c, P, R = st["cache"], st["page"], st["runs"]
    slots = st["slots"]
    T = slots.numel()
    # rows that are no tokens repeat the first one, which is
    row = torch.where(slots >= 0, torch.arange(T, device=DEV), 0)
    slot = slots[row]
    page, off = slot // P, slot % P
    new = torch.ones_like(page, dtype=torch.bool)
    new[1:] = page[1:] != page[:-1]
    new &= slots >= 0
    run = (new.cumsum(0) - 1)[row]
    at = torch.zeros(R, dtype=torch.int64, device=DEV).scatter_(0, run, page)
    o = torch.full((R,), P, device=DEV).scatter_reduce_(0, run, off, "amin")
    end = torch.zeros(R, dtype=torch.int64, device=DEV).scatter_reduce_(0, run, off + 1, "amax")
    H = c["k_scale"].shape[1]
    h = torch.arange(H, device=DEV)[None]
    pos = torch.arange(P, device=DEV)
    for name in ("k", "v"):
        is_k = name == "k"
        x = st[name][row].float()
        fine = torch.isfinite(x)
        mag = torch.where(fine, x, 0.0).abs().amax(2)
        amax = torch.zeros((R, H), device=DEV).scatter_reduce_(0, run[:, None].expand(T, H), mag, "amax")
        scale = c[name + "_scale"]
        e_old = torch.where(o[:, None] > 0, torch.frexp(scale[at])[1] - 1, E_MIN)
        e = torch.maximum(e_old, _scale_of(amax))
        b = _to_f8(torch.where(fine, torch.ldexp(x, -e[run][:, :, None]), math.nan))
        pages = c[name].view(torch.uint8)
        # the page's earlier tokens at the new scale
        old = pages[at]
        old = old if is_k else old.transpose(3, 4).reshape(R, H, P, D)
        less = _to_f8(torch.ldexp(old.view(F8).float(), (e_old - e)[:, :, None, None]))
        keep = torch.where((pos < o[:, None])[:, None, :, None] & (e > e_old)[:, :, None, None], less, old)
        pages[at] = keep if is_k else keep.view(R, H, P // 64, 64, D).transpose(3, 4)
        if is_k:
            pages[page[:, None], h, off[:, None]] = b
        else:
            pages[page[:, None], h, (off // 64)[:, None], :, (off % 64)[:, None]] = b
        scale[at] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
        if is_k:
            val = pages[at].view(F8).double() * (pos < end[:, None])[:, None, :, None]
            c["k_sum"][at] = (val.sum(2) * scale[at].double()[..., None]).float()
    return c


def _plain_decode(st):
    c, P, q = st["cache"], st["page"], st["q"].float()
    lens, block, topk = st["lens"].long(), st["block"], st["topk"]
    S, Hq = q.shape[:2]
    H = c["k_scale"].shape[1]
    G = Hq // H
    idx = st["table"].long()
    W = idx.shape[1]
    n = W * P
    q = q.view(S, H, G, D)
    pos = torch.arange(n, device=DEV)
    use = (pos < lens[:, None])[:, None, None]
    if topk:
        per = block // P
        nb = _ceil(W, per)
        pad = torch.nn.functional.pad(idx, (0, nb * per - W))
        sums = c["k_sum"][pad].double().view(S, nb, per, H, D).sum(2)
        score = torch.matmul(q.double(), sums.permute(0, 2, 3, 1).contiguous())  # [S, H, G, nb]
        cur = ((lens - 1).clamp(min=0) // block).view(S, 1, 1, 1)
        j = torch.arange(nb, device=DEV)
        score = torch.where(j < cur, score, -math.inf)
        order = score.sort(dim=-1, descending=True, stable=True).indices  # equal scores: lower block
        kept = torch.zeros_like(score, dtype=torch.bool).scatter_(-1, order, (j < topk - 1).expand_as(score).contiguous())
        kept = (kept & (j < cur)) | (j == cur)
        use = use & kept[..., pos // block]
    def take(x, scale):
        return x.view(torch.uint8)[idx].view(F8).float() * scale[idx].view(S, W, H, *[1] * (x.dim() - 2))
    K = take(c["k"], c["k_scale"]).permute(0, 2, 1, 3, 4).reshape(S, H, n, D)
    logit = torch.matmul(q, K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    del K
    logit = torch.where(use, logit, -math.inf)
    m = logit.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(logit - m)
    del logit
    l = p.sum(-1, keepdim=True)
    V = take(c["v"], c["v_scale"]).permute(0, 2, 1, 3, 5, 4).reshape(S, H, n, D)
    o = torch.matmul(p, V) / torch.where(l > 0, l, 1.0)
    lse = torch.log(l) + m
    return {"out": o.view(S, Hq, D).to(torch.bfloat16), "lse": lse.view(S, Hq).t().contiguous()}


def run(state):
    op = state["op"]
    if not own:
        return {"plan": _plain_plan, "write": _plain_write, "decode": _plain_decode}[op](state)
    from paper_2502_13189_amd import binding
    if op == "plan":
        p = binding.cache_plan(state["add"], state["lens"], state["table"], state["free"],
                               state["num_free"], state["page"], state["tokens"])
        return {"cu": p.cu_new, "slots": p.slots, "lens": p.lens, "num_free": p.num_free,
                "table": state["table"], "free": state["free"], "refused": p.refused}
    cache = binding.PagedCache(**state["cache"])
    if op == "write":
        binding.cache_write(state["k"], state["v"], state["slots"], cache)
        return state["cache"]
    out, lse = binding.cache_decode(state["q"], cache, state["table"], state["lens"],
                                    state["block"], state["topk"])
    return {"out": out, "lse": lse}


def _distinct(case, L):
    """Tokens of a request's cache that a MoBA call reads for a kv-head, at least: topk blocks
    (its query heads may choose more between them)."""
    B = case["block"]
    c = (L - 1) // B
    return min(case["topk"] - 1, c) * B + L - c * B


def work(case):
    op, P, lens = case["op"], case["page"], _ints(case["lens"])
    H, S = case["hkv"], len(lens)
    if op != "decode":
        add = _ints(case["add"])
        T = sum(max(a, 0) for a in add)
        pages = sum(_ceil(x + a, P) - _ceil(x, P) if a > 0 else _ceil(x, P) if a < 0 else 0 for x, a in zip(lens, add))
        if op == "plan":
            return {"bytes": 16 * S + 8 * T + 8 * pages, "flops": 0}
        el = 4 if case["dtype"] == "f32" else 2
        runs = sum(_ceil(x + a, P) - x // P for x, a in zip(lens, add) if a)
        old = sum(x % P for x, a in zip(lens, add) if a)  # earlier keys of the page: for its sum
        return {"bytes": 8 * T + H * (T * D * 2 * (el + 1) + runs * (16 + 4 * D) + old * D),
                "flops": H * T * D * 6}
    full = not case["topk"]
    keys = sum(L if full else _distinct(case, L) for L in lens if L)
    gate = 0 if full else sum(L // P * D * 4 for L in lens)
    return {"bytes": H * (keys * 2 * D + gate) + S * case["hq"] * D * 4, "flops": 4 * D * case["hq"] * keys}


# ------------------------------------------------------------------ 64 bits
def _f8_values():
    """The finite values of e4m3, ascending."""
    v = [0.0] + [m * 2.0 ** -9 for m in range(1, 8)]
    v += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
    return torch.tensor([-x for x in v[:0:-1]] + v, dtype=torch.float64, device=DEV)


def _round_f8(x, vals):
    """The nearest e4m3 value (ties to the even code), of numbers within its range."""
    hi = torch.searchsorted(vals, x.contiguous()).clamp(max=vals.numel() - 1)
    lo = (hi - 1).clamp(min=0)
    a, b = vals[lo], vals[hi]
    zero = vals.numel() // 2  # a value's code is its distance from 0
    up = (b - x < x - a) | ((b - x == x - a) & ((hi - zero) % 2 == 0))
    return torch.where(up, b, a)


def _exact_plan(case, st):
    add, lens, P = _ints(case["add"]), _ints(case["lens"]), case["page"]
    table, free = st["table"].cpu().numpy().copy(), st["free"].cpu().numpy().copy()
    n, W, T = int(st["num_free"]), table.shape[1], st["tokens"]
    for s, a in enumerate(add):
        if a < 0:
            m = _ceil(lens[s], P)
            free[n:n + m] = table[s, :m]
            n += m
    slots = torch.full((T,), -1, dtype=torch.int64)
    cu, new, refused, full = [0], [], 0, False
    for s, a in enumerate(add):
        t0, t1 = cu[-1], cu[-1] + max(a, 0)
        cu.append(t1)
        h, need = _ceil(lens[s], P), _ceil(lens[s] + max(a, 0), P) - _ceil(lens[s], P)
        if a < 0:
            new.append(0)
            continue
        fits = h + need <= W and t1 <= T
        full |= fits and need > n
        if not fits or (full and need):
            refused += 1
            new.append(lens[s])
            continue
        for j in range(h, h + need):
            n -= 1
            table[s, j] = free[n]
        pos = torch.arange(lens[s], lens[s] + a)
        slots[t0:t1] = torch.from_numpy(table[s])[pos // P].long() * P + pos % P
        new.append(lens[s] + a)
    i32 = dict(dtype=torch.int32)
    return {"cu": torch.tensor([min(x, T) for x in cu], **i32), "slots": slots, "lens": torch.tensor(new, **i32),
            "num_free": torch.tensor([n], **i32), "table": torch.from_numpy(table),
            "free": torch.from_numpy(free), "refused": torch.tensor([refused], **i32)}


def _exact_write(case, st):
    vals, P = _f8_values(), case["page"]
    c = st["cache"]
    out = {"k_sum": c["k_sum"].double()}
    slots = st["slots"].tolist()
    runs = []
    for t, s in enumerate(slots):
        if s >= 0 and (t == 0 or slots[t - 1] != s - 1 or s % P == 0):
            runs.append([t, s, 1])
        elif s >= 0:
            runs[-1][2] += 1
    for name in ("k", "v"):
        old = c[name].double()
        if name == "v":  # [N, H, P / 64, D, 64] -> [N, H, P, D]
            old = old.transpose(3, 4).reshape(old.shape[0], old.shape[1], P, D)
        scale = c[name + "_scale"].double().clone()
        x = st[name].double()
        for t, s, m in runs:
            at, o = s // P, s % P
            y = x[t:t + m].transpose(0, 1)  # [H, m, D]
            e = torch.ceil(torch.log2(y.abs().amax((1, 2)) / 448.0)).clamp(E_MIN, E_MAX)
            if o:
                was = torch.log2(scale[at])
                e = torch.maximum(e, was)
                old[at, :, :o] = _round_f8(old[at, :, :o] * torch.exp2(was - e)[:, None, None], vals)
            scale[at] = torch.exp2(e)
            old[at, :, o:o + m] = _round_f8(y * torch.exp2(-e)[:, None, None], vals)
            if name == "k":
                out["k_sum"][at] = old[at, :, :o + m].sum(1) * scale[at][:, None]
        out[name + "_scale"] = scale
        out[name] = old if name == "k" else old.view(*old.shape[:2], P // 64, 64, D).transpose(3, 4)
    return out


def _exact_decode(case, st):
    c, P, B = st["cache"], case["page"], case["block"]
    H, Hq, topk = case["hkv"], case["hq"], case["topk"]
    G, lens = Hq // H, _ints(case["lens"])
    out = torch.zeros((len(lens), Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((Hq, len(lens)), -math.inf, dtype=torch.float64, device=DEV)
    for s, L in enumerate(lens):
        if not L:
            continue
        at = st["table"][s, :_ceil(L, P)].long()
        for g in range(H):
            q = st["q"][s, g * G:(g + 1) * G].double()
            k = c["k"].view(torch.uint8)[at, g].view(F8).double() * c["k_scale"][at, g].double()[:, None, None]
            v = c["v"].view(torch.uint8)[at, g].view(F8).double() * c["v_scale"][at, g].double()[:, None, None, None]
            k = k.reshape(-1, D)[:L]
            v = v.transpose(2, 3).reshape(-1, D)[:L]
            z = (q @ k.t()) / math.sqrt(D)
            if topk:
                cur = (L - 1) // B
                per = B // P
                sums = c["k_sum"][at[:cur * per], g].double().view(cur, per, D).sum(1)
                for h, sc in enumerate((q @ sums.t()).tolist()):
                    best = sorted(range(cur), key=lambda j: (-sc[j], j))[:topk - 1]
                    drop = torch.ones(cur + 1, dtype=torch.bool, device=DEV)
                    drop[best + [cur]] = False
                    z[h][drop.repeat_interleave(B)[:L]] = -math.inf
            lse[g * G:(g + 1) * G, s] = torch.logsumexp(z, 1)
            out[s, g * G:(g + 1) * G] = torch.softmax(z, 1) @ v
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    return {"plan": _exact_plan, "write": _exact_write, "decode": _exact_decode}[case["op"]](case, st)
