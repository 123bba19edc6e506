"""The operators of the 4-bit key/value cache, case by case: plain forms and calls.

The cache holds the keys and values of an agent's context in pages: blocks of 32
channels of one token of one key/value head, each with 4-bit codes (sign and the
magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6) and one power-of-two scale.  Operators:

  append   K and V rows into the pages of ragged sequences (``kv_append``), and the
           values that the cache then stands for (``kv_read``)
  attend   attention of single tokens or chunks of queries over the cache, with
           grouped heads, a causal limit or a mask of slots, and on request the
           attention weight that each cached token received (``kv_attend``)
  evict    a cache over its budget brought back to it: the slots of the largest
           accumulated weights stay, the newest and the first are protected
           (``kv_evict``)

One head's part of a page of T tokens and D channels is, in bytes: K codes
[T][D/2], V codes [T/4][16][4][D/32] (16 runs of D/16 channels, four tokens at a
time), K scales [T][D/32], V scales [T/4][D/32][4].

``own`` false: elementary torch operations in float32; true: the library's calls.
``exact`` gives the outputs in float64.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32                       # channels that share a scale
E_LO, E_HI = -23, 13             # exponents of the scales
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # a decode step writes one token for each of four agents
        dict(name="append_step", op="append", B=4, n=1, L=1000, Hk=8, D=128, T=64, dt="bf16", ragged=False),
        # prompts of different lengths enter the cache
        dict(name="append_prompts", op="append", B=5, n=5003, L=5003, Hk=8, D=128, T=64, dt="bf16", ragged=True),
        # a retrieval batch's contexts enter the cache
        dict(name="append_bulk", op="append", B=16, n=8192, L=8192, Hk=8, D=128, T=64, dt="f16", ragged=False),
        # the first token after one retrieved record of 47 tokens: the latency of a call
        dict(name="decode_first", op="attend", B=1, n=1, L=47, Hq=32, Hk=8, D=128, T=64, dt="bf16", ragged=False,
             causal=True, mask=False, weights=False),
        # a decode step of 37 agents at different points of their trajectories, seven heads a group
        dict(name="decode_agents", op="attend", B=37, n=1, L=6000, Hq=28, Hk=4, D=128, T=64, dt="bf16", ragged=True,
             causal=True, mask=False, weights=False),
        # the longest contexts: eight sequences of 131,072 tokens
        dict(name="decode_long", op="attend", B=8, n=1, L=131072, Hq=32, Hk=8, D=128, T=64, dt="bf16", ragged=False,
             causal=True, mask=False, weights=False),
        # a decode step of a bounded cache: the weights that eviction goes by
        dict(name="decode_weights", op="attend", B=16, n=1, L=16383, Hq=32, Hk=8, D=128, T=64, dt="f16", ragged=True,
             causal=True, mask=False, weights=True),
        # three queries a sequence over a window of 512 tokens of which a mask takes some out, one head a group
        dict(name="window_mask", op="attend", B=64, n=3, L=512, Hq=12, Hk=12, D=64, T=32, dt="f16", ragged=False,
             causal=False, mask=True, weights=False),
        # a chunk of a long prompt against all that came before
        dict(name="chunk_prompt", op="attend", B=1, n=2048, L=32768, Hq=32, Hk=8, D=128, T=64, dt="bf16", ragged=False,
             causal=True, mask=False, weights=False),
        # chunks of several prompts, with weights
        dict(name="chunk_weights", op="attend", B=6, n=513, L=4099, Hq=16, Hk=4, D=64, T=128, dt="f16", ragged=True,
             causal=True, mask=False, weights=True),
        # a cache that is one token over its budget, every decode step
        dict(name="evict_step", op="evict", B=8, L=4097, budget=4096, recent=512, sinks=4, Hk=8, D=128, T=64),
        # prompts cut to a quarter after they were read
        dict(name="evict_prompts", op="evict", B=24, L=32768, budget=8192, recent=1024, sinks=4, Hk=8, D=128, T=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "decode", "chunk", "chunk", "evict"])
    D = rng.choice([64, 128, 128, 256])
    T = rng.choice([32, 64, 64, 128, 256])
    Hk = rng.choice([1, 2, 4, 8, 8, 12])
    dt = rng.choice(["bf16", "f16"])
    tokens = 8 * 131072 * 8 * 128 // (Hk * D)              # tokens of the largest cache
    if op == "append":
        B = _log_int(rng, 1, 32)
        n = 1 if rng.random() < 0.3 else _log_int(rng, 1, max(1, min(16384, tokens // 8 // B)))
        return dict(op="append", B=B, n=n, L=n + rng.choice([0, 0, 1, 777]), Hk=Hk, D=D, T=T, dt=dt,
                    ragged=B > 1 and rng.random() < 0.5)
    if op == "evict":
        B = _log_int(rng, 1, 24)
        L = _log_int(rng, 64, min(65536, tokens // B))
        budget = max(1, min(L - 1, int(L * rng.choice([0.1, 0.25, 0.5, 0.9, 0.999]))))
        recent = int(budget * rng.choice([0.0, 0.1, 0.25]))
        return dict(op="evict", B=B, L=L, budget=budget, recent=recent, sinks=min(budget - recent, rng.choice([0, 1, 4])),
                    Hk=Hk, D=D, T=T)
    G = rng.choice([1, 2, 4, 4, 7, 8, 16])
    mask, weights = rng.random() < 0.25, rng.random() < 0.35
    if op == "decode":
        B = _log_int(rng, 1, 64)
        L = _log_int(rng, 1, min(131072, tokens // B))
        return dict(op="attend", B=B, n=rng.choice([1, 1, 1, 2, 4]) if L >= 4 else 1, L=L, Hq=G * Hk, Hk=Hk, D=D, T=T,
                    dt=dt, ragged=B > 1 and rng.random() < 0.5, causal=rng.random() < 0.7, mask=mask, weights=weights)
    B = _log_int(rng, 1, 8)
    L = _log_int(rng, 64, 32768)
    most = 32 * 2048 * 32768 * 128 // (B * G * Hk * L * D * 2)
    n = _log_int(rng, 8, max(8, min(L, 2048, most)))
    return dict(op="attend", B=B, n=n, L=L, Hq=G * Hk, Hk=Hk, D=D, T=T, dt=dt, ragged=B > 1 and rng.random() < 0.5,
                causal=rng.random() < 0.8, mask=mask, weights=weights)


# ------------------------------------------------------------------ sizes of a case
def _sizes(case):
    """Rows and lengths of each sequence: equal, or falling from the case's to about half of it."""
    B, n, L = case["B"], case.get("n", 1), case["L"]
    if not case.get("ragged"):
        return [n] * B, [L] * B
    rows = [n - (b * (n // 2)) // B for b in range(B)]
    return rows, [max(r, L - (b * (L // 2)) // B) for b, r in enumerate(rows)]


def work(case):
    D, Hk = case["D"], case["Hk"]
    token = Hk * (D + D // 16)                                       # bytes of a cached token
    if case["op"] == "evict":
        B, L, keep = case["B"], case["L"], case["budget"]
        moved = (L - keep) * keep / L                                # kept tokens beyond the budget
        return dict(bytes=B * (Hk * (8.0 * L + 12.0 * keep) + 2 * moved * token), flops=0)
    rows, lens = _sizes(case)
    if case["op"] == "append":                                       # rows in, codes out, codes in, values out
        return dict(bytes=float(sum(rows)) * (8 * Hk * D + 2 * token), flops=0)
    seen = sum(r * l - (r * (r - 1) // 2 if case["causal"] else 0) for r, l in zip(rows, lens))
    size = sum(lens) * token + 4 * sum(rows) * case["Hq"] * D + sum(lens) * (case["mask"] + 8 * Hk * case["weights"])
    return dict(bytes=float(size), flops=4.0 * seen * case["Hq"] * D)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _quantize(x):
    """Codes (uint8, one per value) and scale exponents of the blocks of x (last axis)."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    amax = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, torch.where(m <= 0.75, e - 3, e - 2), E_LO).clamp(E_LO, E_HI)
    y = torch.ldexp(x.abs(), -e)
    code = (y > 0.25).to(torch.uint8)                                # halfway goes to the even code
    for t, up in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (y >= t) if up else (y > t)
    return (code | ((x < 0).to(torch.uint8) << 3)).flatten(-2), e.squeeze(-1)


def _pack_pages(k, v):
    """Pages [n, Hk, bytes] of k, v [n, Hk, T, D]."""
    n, Hk, T, D = k.shape
    (kc, ke), (vc, ve) = _quantize(k), _quantize(v)
    kb, vb = (c[..., 0::2] | (c[..., 1::2] << 4) for c in (kc, vc))
    ks, vs = ((e + 127).to(torch.uint8) for e in (ke, ve))
    vb = vb.view(n, Hk, T // 4, 4, 16, D // 32).transpose(3, 4)
    vs = vs.view(n, Hk, T // 4, 4, D // 32).transpose(3, 4)
    return torch.cat([t.reshape(n, Hk, -1) for t in (kb, vb, ks, vs)], dim=-1)


def _rows(g, n, heads, D, dt, spread=None):
    """Rows of a key, value or query projection; keys have channels of different sizes."""
    x = torch.randn((n, heads, D), generator=g, device="cuda")
    return (x if spread is None else x * spread).to(dt)


def _cache(g, case, filled):
    """A pool of pages for the case's sequences, in an order of its own, and its table."""
    B, Hk, D, T = case["B"], case["Hk"], case["D"], case["T"]
    per = -(-case["L"] // T)
    pages = B * per + 3
    pool = torch.zeros((pages, Hk, T * (D + D // 16)), dtype=torch.uint8, device="cuda")
    table = torch.randperm(pages, generator=g, device="cuda")[: B * per].view(B, per).to(torch.int32)
    if filled:
        spread = torch.exp(0.5 * torch.randn((Hk, 1, D), generator=g, device="cuda"))
        step = max(1, (1 << 26) // (Hk * T * D))
        for at in range(0, pages, step):
            n = min(step, pages - at)
            k, v = (torch.randn((n, Hk, T, D), generator=g, device="cuda") for _ in range(2))
            pool[at:at + n] = _pack_pages((k * spread).half(), v.half())
    return pool, table


def prepare(case, seed):
    g = _gen(seed)
    B, Hk, D = case["B"], case["Hk"], case["D"]
    rows, lens = _sizes(case)
    s = dict(case=case, lengths=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    s["pool"], s["table"] = _cache(g, case, case["op"] != "append")
    if case["op"] == "evict":
        L = case["L"]
        # accumulated weights: a few tokens hold most of the mass; older ones had longer to gather it
        w = torch.exp(1.5 * torch.randn((B, Hk, L), generator=g, device="cuda"))
        s["scores"] = w * torch.linspace(2.0, 0.5, L, device="cuda")
        # the positions that survived earlier evictions, in any order, then the newest in order
        old = min(case["budget"], L - 1)
        pos = torch.argsort(torch.rand((B, Hk, old), generator=g, device="cuda"), dim=-1).to(torch.int32) * 2
        new = 2 * old + torch.arange(L - old, dtype=torch.int32, device="cuda").expand(B, Hk, L - old)
        s["positions"] = torch.cat([pos, new], dim=-1).contiguous()
        return s
    total = sum(rows)
    s["starts"] = None
    if case["ragged"]:
        s["starts"] = torch.tensor([sum(rows[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    s["left"] = torch.tensor(rows, device="cuda")                    # rows of each sequence
    s["seq"] = torch.repeat_interleave(torch.arange(B, device="cuda"), s["left"])
    first = s["left"].cumsum(0) - s["left"]                          # sequence and place of every row
    s["place"] = torch.arange(total, device="cuda") - first[s["seq"]]
    dt = DT[case["dt"]]
    if case["op"] == "append":
        spread = torch.exp(0.5 * torch.randn((Hk, D), generator=g, device="cuda"))
        s["k"], s["v"] = _rows(g, total, Hk, D, dt, spread), _rows(g, total, Hk, D, dt)
        return s
    s["q"] = _rows(g, total, case["Hq"], D, dt)
    s["mask"] = None
    if case["mask"]:                                                 # records of 16 tokens, a quarter of them left out
        records = -(-case["L"] // 16)
        s["mask"] = (torch.rand((B, 1, records), generator=g, device="cuda") > 0.25).repeat_interleave(16, dim=-1)[..., : case["L"]].contiguous()
    s["weights"] = None
    if case["weights"]:
        s["weights"] = torch.rand((B, Hk, case["L"]), generator=g, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms
def _magnitudes():
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")


def _unpack(pool, D, T):
    """Values (k, v) [..., T, D] in float32 of pages [..., bytes]."""
    lead, cut = pool.shape[:-1], T * D // 2
    kb, vb, ks, vs = pool.split([cut, cut, T * D // 32, T * D // 32], dim=-1)
    vb = vb.reshape(*lead, T // 4, 16, 4, D // 32).transpose(-2, -3)
    vs = vs.reshape(*lead, T // 4, D // 32, 4).transpose(-1, -2)
    m = _magnitudes()
    signed = torch.cat([m, -m])
    byte = torch.arange(256, device="cuda")
    pairs = torch.stack([signed[byte & 15], signed[byte >> 4]], dim=-1)      # the two values of a byte

    def values(b, e):
        x = pairs.index_select(0, b.reshape(-1).int()).view(*lead, T, D // BLOCK, BLOCK)
        return (x * torch.exp2(e.reshape(*lead, T, D // BLOCK, 1).float() - 127.0)).flatten(-2)

    return values(kb, ks), values(vb, vs)


def _gathered(s):
    """K and V [B, Hk, slots, D] in float32 of the case's sequences."""
    c = s["case"]
    k, v = _unpack(s["pool"][s["table"].long()], c["D"], c["T"])             # [B, pages, Hk, T, D]
    return k.transpose(1, 2).flatten(2, 3), v.transpose(1, 2).flatten(2, 3)


def _plain_append(s):
    c, T, D = s["case"], s["case"]["T"], s["case"]["D"]
    seq, place, Hk = s["seq"], s["place"], c["Hk"]
    slot = s["lengths"].long()[seq] - s["left"][seq] + place
    page, at = s["table"].long()[seq, slot // T], slot % T
    cut = T * D // 2
    pool = s["pool"]
    h = torch.arange(Hk, device="cuda")[None, :, None]
    p, t = page[:, None, None], at[:, None, None]
    out = []
    for x, first, scales in ((s["k"], 0, 2 * cut), (s["v"], cut, 2 * cut + T * D // 32)):
        code, e = _quantize(x)
        byte = code[..., 0::2] | (code[..., 1::2] << 4)                      # [rows, Hk, D/2]
        j, b = torch.arange(D // 2, device="cuda"), torch.arange(D // 32, device="cuda")
        if first == 0:
            jj, bb = t * (D // 2) + j, t * (D // 32) + b
        else:
            run = D // 32
            jj = ((t // 4 * 16 + j // run) * 4 + t % 4) * run + j % run
            bb = (t // 4 * run + b) * 4 + t % 4
        pool[p, h, first + jj] = byte
        pool[p, h, scales + bb] = (e + 127).to(torch.uint8)
        m = _magnitudes()[(code & 7).long()]
        m = torch.where(code >= 8, -m, m).unflatten(-1, (-1, BLOCK))
        out.append((m * torch.exp2(e.float())[..., None]).flatten(-2).to(x.dtype))
    return dict(k=out[0], v=out[1])


def _plain_attend(s):
    c = s["case"]
    B, Hk, D, G, n = c["B"], c["Hk"], c["D"], c["Hq"] // c["Hk"], c["n"]
    k, v = _gathered(s)
    S = k.shape[2]
    seq, place = s["seq"], s["place"]
    q = torch.zeros((B, n, Hk, G, D), device="cuda")
    q[seq, place] = s["q"].float().view(-1, Hk, G, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hk, n * G, D)
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(D ** -0.5).view(B, Hk, n, G, S)
    slot = torch.arange(S, device="cuda")
    lens = s["lengths"].long()
    end = lens[:, None].expand(B, n)
    if c["causal"]:
        end = end - s["left"][:, None] + 1 + torch.arange(n, device="cuda")
    seen = (slot < torch.minimum(end, lens[:, None])[..., None])[:, None, :, None, :]
    if s["mask"] is not None:
        seen = seen & torch.nn.functional.pad(s["mask"], (0, S - s["mask"].shape[-1]))[:, :, None, None, :]
    x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    o = torch.matmul(p.view(B, Hk, n * G, S), v).view(B, Hk, n, G, D).permute(0, 2, 1, 3, 4)
    out = dict(out=o[seq, place].reshape(-1, c["Hq"], D).to(s["q"].dtype))
    if s["weights"] is not None:
        there = (torch.arange(n, device="cuda") < s["left"][:, None])[:, None, :, None, None]
        w = torch.where(there, p, torch.zeros_like(p)).sum((2, 3))
        out["weights"] = s["weights"].add_(w[..., : s["weights"].shape[-1]])
    return out


def _plain_evict(s):
    c = s["case"]
    D, T, keep, L = c["D"], c["T"], c["budget"], c["L"]
    slot = torch.arange(L, device="cuda")
    pos, w = s["positions"], s["scores"]
    there = slot < s["lengths"].long()[:, None, None]
    newest = pos.gather(-1, (s["lengths"].long() - 1)[:, None, None].expand(-1, c["Hk"], 1))
    safe = (pos < c["sinks"]) | (pos > newest - c["recent"])
    key = torch.where(safe, torch.full_like(w, math.inf), w)
    key = torch.where(there, key, torch.full_like(w, -math.inf))
    chosen = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    stays = torch.zeros_like(there.expand_as(key)).scatter_(-1, chosen, True)
    hole, extra = ~stays[..., :keep], stays[..., keep:]
    # the i-th hole takes the i-th slot kept beyond the budget
    rank = hole.cumsum(-1) - 1
    late = torch.argsort((~extra).to(torch.uint8), dim=-1, stable=True) + keep
    late = torch.nn.functional.pad(late, (0, max(0, keep - late.shape[-1])))
    kept = torch.where(hole, late.gather(-1, rank.clamp(min=0)), slot[:keep])
    # move the tokens' bytes
    table, pool = s["table"].long(), s["pool"]
    b, h, at = hole.nonzero(as_tuple=True)
    src = kept[b, h, at]
    cut, run = T * D // 2, D // 32
    j, g = torch.arange(D // 2, device="cuda"), torch.arange(run, device="cuda")

    def places(t):
        t = (t % T)[:, None]
        return torch.cat([t * (D // 2) + j, cut + ((t // 4 * 16 + j // run) * 4 + t % 4) * run + j % run,
                          2 * cut + t * run + g, 2 * cut + T * run + (t // 4 * run + g) * 4 + t % 4], dim=1)

    ps, pd, hh = table[b, src // T][:, None], table[b, at // T][:, None], h[:, None]
    pool[pd, hh, places(at)] = pool[ps, hh, places(src)]
    return dict(kept=kept.to(torch.int32), scores=w.gather(-1, kept), positions=pos.gather(-1, kept),
                lengths=s["lengths"].clamp(max=keep), cache=pool)


def run(s):
    c = s["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[c["op"]](s)
    import paper_2609_32256_amd as lam
    if c["op"] == "append":
        lam.kv_append(s["k"], s["v"], s["pool"], s["table"], s["lengths"], starts=s["starts"])
        k, v = lam.kv_read(s["pool"], s["table"], s["lengths"], s["k"].shape[0], c["D"], dtype=s["k"].dtype, starts=s["starts"])
        return dict(k=k, v=v)
    if c["op"] == "attend":
        o = lam.kv_attend(s["q"], s["pool"], s["table"], s["lengths"], starts=s["starts"], causal=c["causal"],
                          mask=s["mask"], weights=s["weights"], max_length=c["L"])
        return dict(out=o) if s["weights"] is None else dict(out=o, weights=s["weights"])
    kept, scores, positions, lengths = lam.kv_evict(s["pool"], s["table"], s["lengths"], s["scores"], c["budget"], c["D"],
                                                    recent=c["recent"], sinks=c["sinks"], positions=s["positions"])
    return dict(kept=kept, scores=scores, positions=positions, lengths=lengths, cache=s["pool"])


# ------------------------------------------------------------------ outputs in 64 bits
_VALUE = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_head(s, b, h):
    """K and V [slots, D] in float64 of one sequence's head, read code by code."""
    c = s["case"]
    D, T = c["D"], c["T"]
    raw = s["pool"][s["table"][b].long(), h].long()                          # [pages, bytes]
    lut = torch.tensor(_VALUE + [-x for x in _VALUE], dtype=torch.float64, device="cuda")
    t, d = torch.meshgrid(torch.arange(T, device="cuda"), torch.arange(D, device="cuda"), indexing="ij")
    run = D // 16
    kat = t * (D // 2) + d // 2
    vat = T * D // 2 + (((t // 4) * 16 + d // run) * 4 + t % 4) * (run // 2) + (d % run) // 2
    kst = T * D + t * (D // 32) + d // 32
    vst = T * D + T * (D // 32) + ((t // 4) * (D // 32) + d // 32) * 4 + t % 4
    out = []
    for at, st in ((kat, kst), (vat, vst)):
        code = (raw[:, at] >> (4 * (d % 2))) & 15
        out.append((lut[code] * torch.pow(2.0, (raw[:, st] - 127).double())).flatten(0, 1))
    return out


def _exact_values(x):
    """The nearest representable value of every element, by trying all eight."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(amax, E_LO)
    for k in range(E_LO, E_HI):
        e = torch.where(amax > 6.0 * 2.0 ** k, torch.full_like(e, k + 1), e)
    y = x.abs() * torch.pow(2.0, -e)
    best, err = torch.zeros_like(y), y.clone()
    for i, m in enumerate(_VALUE[1:], 1):
        d = (y - m).abs()
        take = (d < err) | ((d == err) & (i % 2 == 0))
        best, err = torch.where(take, torch.full_like(best, m), best), torch.where(take, d, err)
    return (torch.sign(x) * best * torch.pow(2.0, e)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return dict(k=_exact_values(s["k"]), v=_exact_values(s["v"]))
    if case["op"] == "evict":
        return _exact_evict(s)
    rows, lens = _sizes(case)
    G, D = case["Hq"] // case["Hk"], case["D"]
    out = torch.zeros((sum(rows), case["Hq"], D), dtype=torch.float64, device="cuda")
    weights = None if s["weights"] is None else s["weights"].double()
    at = 0
    for b, (n, L) in enumerate(zip(rows, lens)):
        i, t = torch.arange(n, device="cuda")[:, None], torch.arange(L, device="cuda")[None, :]
        seen = (t <= L - n + i) if case["causal"] else (t >= 0).expand(n, L)
        if s["mask"] is not None:
            seen = seen & s["mask"][b, 0, None, :L]
        for h in range(case["Hk"]):
            k, v = (x[:L] for x in _exact_head(s, b, h))
            for r in range(h * G, h * G + G):
                x = s["q"][at:at + n, r].double() @ k.T / math.sqrt(D)
                x = torch.where(seen, x, torch.full_like(x, -math.inf))
                p = torch.nan_to_num(torch.softmax(x, dim=-1), nan=0.0)
                out[at:at + n, r] = p @ v
                if weights is not None:
                    weights[b, h, :L] += p.sum(0)
        at += n
    return dict(out=out) if weights is None else dict(out=out, weights=weights)


def _exact_evict(s):
    c = s["case"]
    B, Hk, keep = c["B"], c["Hk"], c["budget"]
    w, pos = s["scores"].double().cpu().numpy(), s["positions"].cpu().numpy()
    scores = torch.empty((B, Hk, keep), dtype=torch.float64)
    for b in range(B):
        L = int(s["lengths"][b])
        for h in range(Hk):
            x = w[b, h, :L].copy()
            x[(pos[b, h, :L] < c["sinks"]) | (pos[b, h, :L] > pos[b, h, L - 1] - c["recent"])] = math.inf
            order = sorted(range(L), key=lambda t: (-x[t], t)) if L < 3000 else (-x).argsort(kind="stable")
            chosen = set(int(t) for t in order[:keep])
            late = iter(t for t in range(keep, L) if t in chosen)
            scores[b, h] = torch.tensor([w[b, h, t if t in chosen else next(late)] for t in range(keep)], dtype=torch.float64)
    return dict(kept=None, scores=scores.cuda(), positions=None, lengths=None, cache=None)
