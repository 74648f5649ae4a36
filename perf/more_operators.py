"""Operators that bound and steer a long generation over the 8-bit paged cache, as measurable cases.

Each case is a dict of plain values; `prepare` makes what a program holds
before the call (queries in the layout of the projection that made them, a
filled cache, page tables, masks of drafted trees, the weights accumulated so
far), `run` is one pass through an operator, in elementary torch operations
or, where `own` is true, through the public Python binding, `work` the bytes
and operations the pass cannot do without, `exact` the same result in 64 bits.

Operators (`op`):

* window   attention of each sequence's new tokens over the last `window` keys
           and the first `sinks`;
* tree     attention of drafted tokens that form a tree: each sees what was
           there before and, of the drafts, those that its bit mask names;
* weights  attention over all keys that also adds to every key's accumulated
           weight what the new tokens' probabilities give it;
* evict    of every KV head's keys, the `budget` that stay (first, last and
           heaviest ones), moved together into other pages.

The cache: codes uint8 in blocks of 32 tokens of one head, 4096 bytes each
([pages, heads, blocks per page, ...]); K as [8 chunks of 16 channels][32
tokens][16 channels], V as [128 channels][32 tokens]; scales uint8 E8M0
[pages, heads, blocks per page]; a code is an E4M3 number.  Weights fp32
[pages, heads, tokens per page].
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
BLOCK = 32


def _case(name, op, S, new, past, Hq, Hkv, page, ragged, **more):
    c = dict(op=op, S=S, new=new, past=past, Hq=Hq, Hkv=Hkv, page=page, ragged=ragged, **more)
    return dict(c, name=name) if name else c


def _window(name, S, new, past, Hq, Hkv, page, window, sinks, ragged=False, causal=True):
    return _case(name, "window", S, new, past, Hq, Hkv, page, ragged, window=window, sinks=sinks, causal=causal)


def _tree(name, S, new, past, Hq, Hkv, page, ragged=False):
    return _case(name, "tree", S, new, past, Hq, Hkv, page, ragged)


def _weights(name, S, new, past, Hq, Hkv, page, ragged=False, causal=True):
    return _case(name, "weights", S, new, past, Hq, Hkv, page, ragged, causal=causal)


def _evict(name, S, keys, Hkv, page, budget, sinks, recent, ragged=False):
    return _case(name, "evict", S, 0, keys, Hkv, Hkv, page, ragged, budget=budget, sinks=sinks, recent=recent)


def listed():
    return [
        # the smallest: one token of one short sequence
        _window("window_tiny", 1, 1, 511, 2, 2, 32, 128, 4),
        # token by token generation far past the window, grouped heads
        _window("window_tokens", 64, 1, 32767, 32, 8, 64, 4096, 4, ragged=True),
        # causal prompts of ragged lengths, several windows long
        _window("window_prompts", 4, 2048, 2048, 32, 8, 128, 1000, 16, ragged=True),
        # the next latent frame of a 480p video over its first frame and the seven frames before it
        _window("window_frame", 1, 1560, 31200, 40, 40, 256, 8 * 1560, 1560, causal=False),
        # a few drafts of one short sequence
        _tree("tree_tiny", 1, 7, 500, 8, 8, 32),
        # trees of 25 drafts of 16 sequences, to be verified at once
        _tree("tree_drafts", 16, 25, 6000, 40, 8, 128, ragged=True),
        # a wide tree over a long context
        _tree("tree_wide", 2, 64, 65536, 32, 8, 256),
        # one token of a short sequence whose keys' weights are kept
        _weights("weights_tiny", 1, 1, 700, 4, 1, 32),
        # token by token generation with the weights that decide about eviction
        _weights("weights_tokens", 64, 1, 8191, 32, 8, 64, ragged=True),
        # prompts of ragged lengths, every key weighed by all tokens behind it
        _weights("weights_prompts", 4, 2048, 2048, 32, 8, 128, ragged=True),
        # 16 sequences of up to 4500 keys, cut to 2048
        _evict("evict_batch", 16, 4500, 8, 64, 2048, 4, 256, ragged=True),
        # one long context cut to an eighth
        _evict("evict_long", 1, 118800, 8, 256, 14850, 64, 1000),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["window", "window", "tree", "weights", "evict"])
    page = rng.choice([32, 64, 128, 256])
    S = _log_int(rng, 1, 64)
    ragged = S > 1 and rng.random() < 0.7
    Hkv = rng.choice([1, 2, 3, 8, 24, 40])
    if op == "evict":
        keys = _log_int(rng, 33, 118800)
        while S * Hkv * keys > 8 * 118800:
            S, keys = (S // 2, keys) if S > 1 else (S, keys // 2)
        budget = max(1, int(keys * rng.uniform(0.05, 0.9)))
        sinks = min(budget, rng.choice([0, 4, rng.randint(1, 100)]))
        return _evict(None, S, keys, Hkv, page, budget, sinks, rng.randint(0, budget - sinks), ragged and S > 1)
    Hq = Hkv * rng.choice([1, 2, 4, 5, 8]) if Hkv < 24 else Hkv
    past = _log_int(rng, 1, 65536) - 1
    if op == "tree":
        new = rng.choice([rng.randint(2, 16), rng.randint(9, 64), _log_int(rng, 33, 200)])
    else:
        new = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 9, 2048)])
    while S * Hkv * (new + past) > 64 * 8 * 8192 or S * Hq * new * (new + past) > 4 * 32 * 2048 * 4096:
        if S > 1:
            S //= 2
        else:
            new, past = max(1, new // 2), past // 2
    ragged = ragged and S > 1
    if op == "tree":
        return _tree(None, S, new, past, Hq, Hkv, page, ragged)
    causal = rng.random() < 0.7
    if op == "weights":
        return _weights(None, S, new, past, Hq, Hkv, page, ragged, causal)
    sinks = rng.choice([0, 4, rng.randint(1, 64), _log_int(rng, 65, 2000)])
    return _window(None, S, new, past, Hq, Hkv, page, _log_int(rng, 32, 16384), sinks, ragged, causal)


# ---------------------------------------------------------------------------
# Inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _lengths(c):
    """New and past tokens of every sequence: those of the case or, ragged, up to those, spread evenly in a mixed order."""
    S, new, past = c["S"], c["new"], c["past"]
    if not c["ragged"]:
        return [new] * S, [past] * S
    share = lambda i, step: 1.0 - 0.9 * (i * step % 1.0)  # noqa: E731
    n = [max(1, round(new * share(i, 0.618034))) for i in range(S)] if new > 8 else [new] * S
    return n, [round(past * share(i, 0.414214)) for i in range(S)]


def _quantized(x):
    """[..., 32 tokens, d] -> E4M3 numbers and E8M0 bytes [...] (the smallest scale that holds the block)."""
    m = x.abs().amax((-2, -1))
    f, e = torch.frexp(m)  # m = f 2^e, 0.5 <= f < 1; 448 = 0.875 * 2^9
    b = torch.where(m > 0, e - 9 + (f > 0.875).to(e.dtype), -127).clamp(-127, 127)
    return torch.ldexp(x, -b[..., None, None]).to(torch.float8_e4m3fn), (b + 127).to(torch.uint8)


def _cache(pages, H, bpp, g):
    """A cache of `pages` pages, filled with keys of heavy tails around a per-head offset, and values whose size
    changes from token to token."""
    kc = torch.empty((pages, H, bpp, 8, BLOCK, 16), dtype=torch.uint8, device="cuda")
    vc = torch.empty((pages, H, bpp, D, BLOCK), dtype=torch.uint8, device="cuda")
    ks = torch.empty((pages, H, bpp), dtype=torch.uint8, device="cuda")
    vs = torch.empty_like(ks)
    offset = math.sqrt(2.0) * torch.randn((H, 1, 1, D), generator=g, device="cuda")
    step = max(1, (1 << 27) // (H * bpp * BLOCK * D))
    for a in range(0, pages, step):
        shape = (min(step, pages - a), H, bpp, BLOCK, D)
        u = torch.rand(shape, generator=g, device="cuda").clamp_(min=1e-7)
        x = torch.randn(shape, generator=g, device="cuda").mul_(torch.rsqrt(u.log_().neg_().add_(0.2))).add_(offset)
        q, ks[a:a + step] = _quantized(x)
        kc[a:a + step] = q.view(torch.uint8).view(*shape[:4], 8, 16).transpose(3, 4)
        size = torch.randn((*shape[:4], 1), generator=g, device="cuda").exp_()
        q, vs[a:a + step] = _quantized(torch.randn(shape, generator=g, device="cuda").mul_(size))
        vc[a:a + step] = q.view(torch.uint8).transpose(3, 4)
    return kc, ks, vc, vs


def _tables(need, order):
    """Page tables [sequences, most pages] of `need` pages each, from `order` on; unused entries -1."""
    table = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for s, k in enumerate(need):
        table[s, :k] = order[at:at + k]
        at += k
    return table.to("cuda")


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _trees(n, words, g):
    """Ancestor masks of random trees: parents among the drafts before, or none (a child of the last certain token)."""
    T = sum(n)
    first = [sum(n[:s]) for s in range(len(n))]
    r = torch.rand((T,), generator=g, device="cuda").cpu().tolist()
    rows = []
    for s, k in enumerate(n):
        mine = []
        for i in range(k):
            parent = int(r[first[s] + i] * (i + 1)) - 1  # -1 .. i - 1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
        rows += mine
    low = (1 << 32) - 1
    signed = lambda x: x - (1 << 32) if x >> 31 else x  # noqa: E731
    return _ints([[signed(m >> 32 * w & low) for w in range(words)] for m in rows])


def prepare(case, seed):
    c, g = case, _generator(seed)
    n, p = _lengths(c)
    L = [a + b for a, b in zip(n, p)]
    page, H = c["page"], c["Hkv"]
    need = [-(-a // page) for a in L]
    kept = [-(-min(a, c["budget"]) // page) for a in L] if c["op"] == "evict" else [0]
    pages = sum(need) + sum(kept) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    st = dict(case=c, table=_tables(need, order), length=_ints(L), cache=_cache(pages, H, page // BLOCK, g), max_kv=max(L))
    if c["op"] in ("weights", "evict"):
        # most keys get little; some nothing
        w = torch.randn((pages, H, page), generator=g, device="cuda").mul_(2.5).exp_()
        w *= torch.rand((pages, H, page), generator=g, device="cuda") > 0.1
        st["weights"] = w
    if c["op"] == "evict":
        return dict(st, to=_tables(kept, order[sum(need):]))
    st.update(start=_ints([sum(n[:s]) for s in range(len(n) + 1)]), max_q=max(n))
    qkv = torch.randn((sum(n), c["Hq"] + 2 * H, D), generator=g, device="cuda").to(torch.bfloat16)  # a projection's output
    st["q"] = qkv[:, :c["Hq"]]
    if c["op"] == "tree":
        st["tree"] = _trees(n, -(-max(n) // 32), g)
    if c["op"] == "weights":
        st["weights_out"] = torch.zeros_like(st["weights"])
    return st


# ---------------------------------------------------------------------------
# One pass


def _views(cache):
    """The cache as the numbers that its bytes stand for."""
    kc, ks, vc, vs = cache
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    return kc.view(f8), ks.view(e8), vc.view(f8), vs.view(e8)


def run(state):
    st, c = state, state["case"]
    op = c["op"]
    if own:
        from paper_2607_24377_amd import mxattn

        if op == "evict":
            kept, count = mxattn.cache_select(st["weights"], st["table"], st["length"], c["budget"], c["sinks"], c["recent"])
            mxattn.cache_compact(*st["cache"], st["table"], kept, count, out_table=st["to"], weights=st["weights"])
            return kept, count, _views(st["cache"]), st["weights"]
        batch = (st["q"], *st["cache"], st["table"], st["start"], st["length"])
        bounds = dict(max_q=st["max_q"], max_kv=st["max_kv"])
        if op == "window":
            return mxattn.cache_attend_window(*batch, c["window"], c["sinks"], c["causal"], **bounds)
        if op == "tree":
            return mxattn.cache_attend_tree(*batch, st["tree"], **bounds)
        return mxattn.cache_attend_weights(*batch, st["weights"], c["causal"], weights_out=st["weights_out"], **bounds)
    if op == "evict":
        return _plain_evict(st)
    return _plain_attend(st)


def _gathered(codes, scales, pages, axes):
    """The numbers of all sequences' pages as fp32, their axes in another order."""
    x = codes[pages].view(torch.float8_e4m3fn).float()  # [S, pages, H, blocks, ...]
    e = scales[pages].int() - 127
    return torch.ldexp(x, e.view(*e.shape, *[1] * (x.dim() - 4))).permute(axes)


def _plain_seen(st, i, j, count, length):
    """[S, n, L]: which keys each new token sees."""
    c = st["case"]
    past = (length - count)[:, None, None]
    own_end = past + i[None, :, None] + 1
    if c["op"] == "tree":
        d = j - past  # [S, 1, L]: which draft a key is
        words = st["tree"].shape[1]
        token = (st["start"].long()[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)  # [S, n]
        word = st["tree"][token].long().gather(2, (d // 32).clamp(0, words - 1).expand(-1, i.numel(), -1))
        bit = (word >> (d % 32)) & 1 == 1
        return (d < 0) | ((d < count[:, None, None]) & bit)
    end = own_end if c["causal"] else length[:, None, None].expand(own_end.shape)
    seen = j < end
    if c["op"] == "window":
        seen = seen & ((j >= end - c["window"]) | (j < c["sinks"]))
    return seen


def _plain_attend(st):
    c, (kc, ks, vc, vs) = st["case"], st["cache"]
    S, Hq, Hkv, page = c["S"], c["Hq"], c["Hkv"], c["page"]
    start, length = st["start"].long(), st["length"].long()
    n, L, G = st["max_q"], -(-st["max_kv"] // page) * page, Hq // Hkv
    pages = st["table"].long().clamp(min=0)
    k = _gathered(kc, ks, pages, (0, 2, 1, 3, 5, 4, 6)).reshape(S, Hkv, L, D)
    v = _gathered(vc, vs, pages, (0, 2, 1, 3, 5, 4)).reshape(S, Hkv, L, D)
    i, j = torch.arange(n, device="cuda"), torch.arange(L, device="cuda")
    count = start[1:] - start[:-1]
    token = (start[:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    real = i < count[:, None]  # [S, n]
    q = st["q"].float()[token].view(S, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, G * n, D)
    seen = _plain_seen(st, i, j, count, length) & real[..., None]
    v = v * (j < length[:, None])[:, None, :, None]
    s = torch.matmul(q, k.transpose(-1, -2)).view(S, Hkv, G, n, L).mul_(1.0 / math.sqrt(D))
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True).clamp(min=1e-38)
    o = torch.matmul(p.view(S, Hkv, G * n, L), v).view(S, Hkv, G, n, D) / l
    o = o.permute(0, 3, 1, 2, 4).reshape(S, n, Hq, D)[real].to(torch.bfloat16)
    if c["op"] != "weights":
        return o
    add = p.div_(l).view(S, Hkv, G * n, L).sum(2)  # [S, Hkv, L]
    before = st["weights"][pages].transpose(1, 2).reshape(S, Hkv, L)
    total = torch.where(j < (length - count)[:, None, None], before, 0.0) + add
    at, head = torch.broadcast_tensors(pages[:, None, j // page], torch.arange(Hkv, device="cuda")[:, None])
    held = (j < length[:, None])[:, None].expand(S, Hkv, L)
    st["weights_out"][at[held], head[held], (j % page).expand(S, Hkv, L)[held]] = total[held]
    return o, st["weights_out"]


def _plain_evict(st):
    c, cache = st["case"], st["cache"]
    S, H, page, budget = c["S"], c["Hkv"], c["page"], c["budget"]
    length, pages = st["length"].long(), st["table"].long().clamp(min=0)
    L = pages.shape[1] * page
    w = st["weights"][pages].transpose(1, 2).reshape(S, H, L)
    j, len3 = torch.arange(L, device="cuda"), length[:, None, None]
    w = torch.where((j < c["sinks"]) | (j >= len3 - c["recent"]), math.inf, w)
    w = torch.where(j < len3, w, -math.inf)
    count = length.clamp(max=budget)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :budget]
    order = torch.nn.functional.pad(order, (0, budget - order.shape[-1]))
    there = torch.arange(budget, device="cuda") < count[:, None, None]
    kept = torch.where(there, order, L).sort(-1).values
    kept = torch.where(there, kept, -1).int()
    # the kept tokens' blocks
    nb = -(-budget // BLOCK)
    src = torch.nn.functional.pad(kept, (0, nb * BLOCK - budget), value=-1).long().view(S, H, nb, BLOCK)
    real, src = src >= 0, src.clamp(min=0)
    seq, head = torch.arange(S, device="cuda")[:, None, None, None], torch.arange(H, device="cuda")[:, None, None]
    pg, blk, slot = pages[seq, src // page], src % page // BLOCK, src % BLOCK
    b = torch.arange(nb, device="cuda")
    bpp = page // BLOCK
    to = st["to"].long()[:, None, (b // bpp).clamp(max=st["to"].shape[1] - 1)].expand(S, H, nb)
    write = (b * BLOCK < count[:, None, None]).expand(S, H, nb)
    at = (to[write], head[..., 0].expand(S, H, nb)[write], (b % bpp).expand(S, H, nb)[write])
    for codes, scales, is_k in ((cache[0], cache[1], True), (cache[2], cache[3], False)):
        was = torch.where(real, scales[pg, head, blk].int(), 0)  # [S, H, nb, 32]
        e = was.amax(-1)
        x = codes[pg, head, blk, :, slot] if is_k else codes[pg, head, blk, :, slot][..., None]
        x = torch.ldexp(x.view(torch.float8_e4m3fn).float(), (was - e[..., None])[..., None, None])
        x = (x * real[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        x = x.transpose(3, 4) if is_k else x[..., 0].transpose(3, 4)
        codes[at] = x[write]
        scales[at] = e.to(torch.uint8)[write]
    moved = st["weights"][pg, head, src % page]
    some = real
    spot = lambda t: t[..., None].expand(S, H, nb, BLOCK)[some]  # noqa: E731
    inside = ((b % bpp * BLOCK)[:, None] + torch.arange(BLOCK, device="cuda")).expand(S, H, nb, BLOCK)
    st["weights"][spot(to), spot(head[..., 0].expand(S, H, nb)), inside[some]] = moved[some]
    return kept, count.int(), _views(cache), st["weights"]


# ---------------------------------------------------------------------------


def _visible(c, n, p):
    """Visible (token, key) pairs of a sequence, and how many of its keys some token sees."""
    L = n + p
    if c["op"] == "window":
        w, a = c["window"], c["sinks"]
        seen = lambda e: e if e <= w + a else w + a  # noqa: E731
        if c["causal"]:
            first = max(0, p + 1 - w)
            return sum(seen(e) for e in range(p + 1, L + 1)), L - max(0, first - a)
        return n * seen(L), seen(L)
    if c["op"] == "tree":
        return round(n * (p + 1 + math.log(n))), L  # (the mean depth of such a tree's nodes)
    return (n * p + n * (n + 1) // 2 if c["causal"] else n * L), L


def work(case):
    c = case
    n, p = _lengths(c)
    if c["op"] == "evict":
        keys, kept = sum(p), sum(min(a, c["budget"]) for a in p)
        return dict(bytes=c["Hkv"] * (4 * keys + kept * (4 * D + 8)), flops=0)
    pairs, keys = (sum(x) for x in zip(*(_visible(c, a, b) for a, b in zip(n, p))))
    held = 8 * c["Hkv"] * keys if c["op"] == "weights" else 0
    return dict(bytes=keys * c["Hkv"] * 2 * D + sum(n) * c["Hq"] * 4 * D + held, flops=4 * pairs * c["Hq"] * D)


# ---------------------------------------------------------------------------
# The same results in 64 bits, sequence by sequence.


def _numbers(codes):
    return codes.view(torch.float8_e4m3fn).double()


def _e4m3(y):
    """Nearest E4M3 number of finite |y| <= 448, ties to even."""
    a = y.abs().clamp(min=2.0 ** -6)
    e = torch.floor(torch.log2(a))
    step = torch.exp2(torch.where(torch.exp2(e) > a, e - 1, e) - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["op"] == "evict":
        return _exact_evict(c, st)
    kc, ks, vc, vs = st["cache"]
    start, length, page = st["start"].tolist(), st["length"].tolist(), c["page"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    G, out = Hq // Hkv, []
    if c["op"] == "weights":
        total = st["weights_out"].double()
    for s in range(c["S"]):
        n, L = start[s + 1] - start[s], length[s]
        pages = st["table"][s, :-(-L // page)].long()
        q = st["q"][start[s]:start[s + 1]].double().view(n, Hkv, G, D)
        t, j = torch.arange(L - n, L, device="cuda")[:, None], torch.arange(L, device="cuda")
        if c["op"] == "tree":
            bits = st["tree"][start[s]:start[s + 1], :, None] >> torch.arange(32, device="cuda", dtype=torch.int32) & 1
            hidden = torch.zeros((n, L), dtype=torch.bool, device="cuda")
            hidden[:, L - n:] = bits.flatten(1)[:, :n] == 0
        else:
            last = t if c["causal"] else torch.full_like(t, L - 1)
            hidden = j > last
            if c["op"] == "window":
                hidden = hidden | ((last - j >= c["window"]) & (j >= c["sinks"]))
        o = torch.empty((n, Hkv, G, D), dtype=torch.float64, device="cuda")
        for h in range(Hkv):
            k = _numbers(kc[pages, h]) * torch.exp2(ks[pages, h].double() - 127)[..., None, None, None]
            k = k.transpose(2, 3).reshape(-1, D)[:L].t().contiguous()
            v = _numbers(vc[pages, h]) * torch.exp2(vs[pages, h].double() - 127)[..., None, None]
            v = v.transpose(2, 3).reshape(-1, D)[:L].contiguous()
            sums = torch.zeros(L, dtype=torch.float64, device="cuda")
            for r in range(G):
                p = torch.softmax((q[:, h, r] @ k / math.sqrt(D)).masked_fill_(hidden, -math.inf), -1)
                p = torch.where(hidden, 0.0, p)
                o[:, h, r] = p @ v
                sums += p.sum(0)
            if c["op"] == "weights":
                sums[:L - n] += st["weights"][pages, h].flatten()[:L - n].double()
                total[pages[j // page], h, j % page] = sums
        out.append(o.view(n, Hq, D))
    return (torch.cat(out), total) if c["op"] == "weights" else torch.cat(out)


def _exact_evict(c, st):
    kc, ks, vc, vs = st["cache"]
    H, page, budget = c["Hkv"], c["page"], c["budget"]
    K, V = _numbers(kc).transpose(3, 4).flatten(4), _numbers(vc).transpose(3, 4).contiguous()  # [..., blocks, 32, d]
    Ke, Ve, W = ks.double() - 127, vs.double() - 127, st["weights"].double()
    length = st["length"].tolist()
    kept = torch.full((c["S"], H, budget), -1, dtype=torch.int32, device="cuda")
    for s, L in enumerate(length):
        pages, to = st["table"][s].long(), st["to"][s].long()
        j = torch.arange(L, device="cuda")
        for h in range(H):
            w = W[pages[j // page], h, j % page]
            if L > budget:
                middle = j[c["sinks"]:L - c["recent"]]
                rank = torch.sort(-w[middle], stable=True).indices[:budget - c["sinks"] - c["recent"]]
                stay = torch.cat((j[:c["sinks"]], middle[rank], j[L - c["recent"]:])).sort().values
            else:
                stay = j
            kept[s, h, :len(stay)] = stay.int()
            at = (pages[stay // page], h, stay % page // BLOCK)
            n, pad = len(stay), -len(stay) % BLOCK
            d = torch.arange(-(-n // BLOCK), device="cuda")
            dst = (to[d * BLOCK // page], h, d * BLOCK % page // BLOCK)
            for X, E in ((K, Ke), (V, Ve)):
                e = E[at]
                top = torch.nn.functional.pad(e, (0, pad), value=-127.0).view(-1, BLOCK).amax(-1)
                x = _e4m3(X[(*at, stay % BLOCK)] * torch.exp2(e - top.repeat_interleave(BLOCK)[:n])[:, None])
                X[dst], E[dst] = torch.nn.functional.pad(x, (0, 0, 0, pad)).view(-1, BLOCK, D), top
            i = torch.arange(n, device="cuda")
            W[to[i // page], h, i % page] = w[stay]
    K = K.unflatten(-1, (8, 16)).transpose(3, 4).contiguous()
    count = st["length"].clamp(max=budget)
    return kept, count, (K, torch.exp2(Ke), V.transpose(3, 4).contiguous(), torch.exp2(Ve)), W
