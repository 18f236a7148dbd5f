"""Rotary positions in front of the paged key/value cache, and the bounding of that cache by accumulated attention weight,
measured.

A case is a dict of plain values; `kind` says which operator it takes:

  rope     T rows of `heads` heads of width hd, the first `rot` channels of each rotated; `style`: pairs (j, j + rot / 2) ("half")
           or (2 j, 2 j + 1) ("interleaved"); `scaling` and `far`: how the frequencies are made for long contexts, and the largest
           position; `x`, `out`: types; `packed`: the rows are columns of one wider tensor
  write    T new tokens: queries rotated, keys rotated and quantized into pages, values quantized into pages
  weights  B sequences, the last `queries` of their tokens as queries: what each token of the cache got of their attention is
           added up per key/value head; `most`, `spread` as for attention ("even", "ragged", "holes"); `fresh`: how many of the newest
           tokens start here ("one", "all")
  evict    B sequences, the most tokens of one `most`: every key/value head keeps `budget` of them, the first `first`, the last
           `recent` and otherwise the heaviest; kept tokens behind the budget move into the holes before it

Codes follow the structure that the method is about: per head a reorder index and four clusters, each with its own scale
and a zero point away from zero.  The position table is the documented one: per position the source channel (int32),
1 / s (fp32), s (fp32), z (int32).
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

CLUSTERS = 4
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token's queries and keys on a 768-wide model's layer: latency and nothing else
        dict(name="rope_t1_24x64", kind="rope", T=1, heads=24, hd=64, rot=64, style="half", scaling="none", far=2048, x="bf16",
             out="bf16", packed=True),
        # several documents in one batch, heads of which a part is rotated, positions far beyond the trained length
        dict(name="rope_t777_25x80_part", kind="rope", T=777, heads=25, hd=80, rot=32, style="interleaved", scaling="parts",
             far=131072, x="f32", out="bf16", packed=False),
        # a long prompt on a 5120-wide layer, out of the projection's output
        dict(name="rope_t8192_80x128", kind="rope", T=8192, heads=80, hd=128, rot=128, style="half", scaling="linear", far=32768,
             x="bf16", out="bf16", packed=True),
        # one token of one sequence
        dict(name="write_t1_12x64_a8", kind="write", T=1, H=12, Hq=12, hd=64, rot=64, style="half", scaling="none", far=2048,
             page=16, bits=8, packed=True),
        # one token of each of 48 sequences, shared key/value heads, half of each head rotated
        dict(name="write_t48_32on8x128_a4", kind="write", T=48, H=8, Hq=32, hd=128, rot=64, style="interleaved", scaling="base",
             far=65536, page=64, bits=4, packed=True),
        # a long prompt on a 5120-wide layer
        dict(name="write_t8192_40x128_a4", kind="write", T=8192, H=40, Hq=40, hd=128, rot=128, style="half", scaling="none",
             far=8192, page=128, bits=4, packed=True),
        # one short sequence on a 768-wide model's layer: latency
        dict(name="weights_b1_l257_12x64_a8", kind="weights", B=1, H=12, Hq=12, hd=64, queries=1, most=257, page=16, bits=8,
             spread="even", fresh="one"),
        # an ordinary serving batch on a 5120-wide layer, one new token per sequence
        dict(name="weights_b32_l4096_40x128_a4", kind="weights", B=32, H=40, Hq=40, hd=128, queries=1, most=4096, page=128, bits=4,
             spread="ragged", fresh="one"),
        # prompts at their end, judged by their last 32 queries; empty sequences and pages that are not here
        dict(name="weights_b5_l8191_32on8x128_q32_a4", kind="weights", B=5, H=8, Hq=32, hd=128, queries=32, most=8191, page=32,
             bits=4, spread="holes", fresh="all"),
        # a serving batch at its budget: a token more, a token less
        dict(name="evict_b32_l2049_8x128_a4", kind="evict", B=32, H=8, hd=128, most=2049, budget=2048, first=4, recent=256, page=64,
             bits=4, spread="even"),
        # wide heads, an odd batch with sequences that are short, empty or partly elsewhere
        dict(name="evict_b7_l1531_2x256_a3", kind="evict", B=7, H=2, hd=256, most=1531, budget=700, first=0, recent=33, page=16,
             bits=3, spread="holes"),
        # long prompts cut down to what will be kept of them
        dict(name="evict_b4_l32768_8x128_a4", kind="evict", B=4, H=8, hd=128, most=32768, budget=4096, first=4, recent=1024, page=128,
             bits=4, spread="ragged"),
    ]


# ---- drawn cases -------------------------------------------------------------------------------------
MOST_ROWS = 8192 * 80 * 128 * 4            # bytes that the largest listed rotation reads and writes
MOST_WRITTEN = 8192 * 5120 * 9             # the same of the largest listed write
MOST_SEEN = 32 * 2048 * 40 * 72            # bytes of keys and weights that the largest listed accumulation goes through
MOST_PAIRS = 5 * 8191 * 32 * 16 * 128      # tokens x heads x queries x width of the one with most queries
MOST_CUT = 4 * 20480 * 8 * 8 + 4 * 8 * 3200 * 256       # bytes of records and rows that the largest listed eviction goes through


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng, hd, most):
    """Key/value heads for up to `most` channels, a multiple of 128 of them."""
    unit = max(1, 128 // hd)
    return max(1, _log_int(rng, 128, most) // (hd * unit)) * unit


def draw(rng):
    kind = rng.choice(["rope", "write", "weights", "weights", "evict", "evict"])
    far = _log_int(rng, 256, 1 << 20)
    turn = dict(style=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "base", "parts"]), far=far)
    if kind == "rope":
        hd = rng.choice([32, 64, 80, 96, 100, 128, 128, 192, 256])
        rot = hd if rng.random() < 0.5 else max(4, int(hd * rng.choice([0.25, 0.4, 0.5])) // 4 * 4)
        heads = _log_int(rng, 1, 96)
        x, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        size = 8 - 2 * (x == "bf16") - 2 * (out == "bf16")
        T = min(_log_int(rng, 1, 32768), MOST_ROWS // (heads * hd * size))
        return dict(kind="rope", T=T, heads=heads, hd=hd, rot=rot, x=x, out=out, packed=rng.random() < 0.5, **turn)
    hd = rng.choice([32, 64, 64, 128, 128, 128, 128, 256])
    bits, page = rng.choice([3, 4, 4, 8]), rng.choice([16, 32, 64, 128, 256])
    if kind == "write":
        H = _heads(rng, hd, 8192)
        share = rng.choice([1, 1, 2, 4, 8])
        while H * share * hd > 12288:
            share = share // 2
        rot = rng.choice([hd, hd, max(16, hd // 2), max(16, hd // 4)])
        T = min(_log_int(rng, 1, 16384), MOST_WRITTEN // (H * hd * (4 * share + 4 + bits // 4)))
        return dict(kind="write", T=T, H=H, Hq=H * share, hd=hd, rot=rot, page=page, bits=bits, packed=rng.random() < 0.5, **turn)
    B = _log_int(rng, 1, 64)
    spread = rng.choice(["even", "ragged", "ragged", "holes"])
    if kind == "weights":
        H = _heads(rng, hd, 8192)
        share = rng.choice([1, 1, 1, 2, 3, 4, 5, 7, 8, 12])
        while H * share * hd > 16384:
            H, share = max(max(1, 128 // hd), H // 2 // max(1, 128 // hd) * max(1, 128 // hd)), max(1, share - 1)
        queries = 1 if rng.random() < 0.6 else _log_int(rng, 2, 64)
        room = min(MOST_SEEN // (B * H * (hd * bits // 8 + 8)), MOST_PAIRS // (B * H * share * hd * queries))
        return dict(kind="weights", B=B, H=H, Hq=H * share, hd=hd, queries=queries, most=_log_int(rng, 1, max(1, min(32768, room))),
                    page=page, bits=bits, spread=spread, fresh=rng.choice(["one", "one", "all"]))
    H = _heads(rng, hd, 2048)
    most = _log_int(rng, 2, max(2, min(65536, MOST_CUT // (B * H * (16 + hd * bits // 8)))))
    budget = most - 1 if rng.random() < 0.3 else _log_int(rng, 1, most)
    first = rng.choice([0, min(4, budget)])
    return dict(kind="evict", B=B, H=H, hd=hd, most=most, budget=budget, first=first,
                recent=rng.choice([0, (budget - first) // 4, budget - first]), page=page, bits=bits, spread=spread)


def _lengths(case):
    """Tokens of every sequence, longest last."""
    B, most = case["B"], case["most"]
    if case["spread"] == "even":
        return [most] * B
    lens = [max(1, most * (i + 1) // B) for i in range(B)]
    if case["spread"] == "holes":
        lens = [0 if i % 3 == 0 and i + 1 < B else n for i, n in enumerate(lens)]
    return lens


def _hole(case, sequence, page_number):
    """Whether that page of that sequence (in the order of _lengths) is not there."""
    if case["spread"] != "holes" or page_number % 5 != 3:
        return False
    return case["kind"] == "weights" or sequence % 3 == 1


# ---- inputs --------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _frequencies(case):
    """(radians per position of every pair in float64, amplitude)."""
    rot, factor, trained = case["rot"], 8.0, 4096.0
    base, amplitude = 10000.0, 1.0
    if case["scaling"] == "base":
        base *= factor ** (rot / max(1, rot - 2))
    f = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        # pairs that turn often over the trained length stay as they are, those that turn less than once are slowed down
        turns = f * trained / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
        amplitude = 0.1 * math.log(factor) + 1.0
    return f, amplitude


def _positions(gen, T, far):
    """A position each of up to 64 sequences, or documents one after the other."""
    if T <= 64:
        return torch.randint(0, far, (T,), generator=gen, device="cuda", dtype=torch.int32)
    starts = torch.randint(0, T, (3,), generator=gen, device="cuda")
    t = torch.arange(T, device="cuda")
    back = torch.where(starts[:, None] <= t, starts[:, None], 0).amax(0)
    begin = int(torch.randint(0, max(1, far - T), (1,), generator=gen, device="cuda"))
    return (t - back + begin).int()


def _position_table(gen, H, hd, bits):
    """[H hd, 4] int32: source channel, 1 / s, s, z of every position (per head: a permutation, four clusters)."""
    d = H * hd
    src = torch.argsort(torch.rand(H, hd, generator=gen, device="cuda"), dim=1) + hd * torch.arange(H, device="cuda")[:, None]
    cluster = (torch.arange(hd, device="cuda") * CLUSTERS // hd).expand(H, hd)
    s = torch.exp(_normal(gen, H, CLUSTERS)).gather(1, cluster).reshape(d) / 2 ** bits
    z = torch.round(_normal(gen, H, CLUSTERS) * 2 ** bits).gather(1, cluster).reshape(d)
    inv_s = (1.0 / s.double()).float()
    return torch.stack([src.reshape(d).int(), inv_s.view(torch.int32), s.view(torch.int32), z.int()], dim=1).contiguous()


def _pack(codes, bits):
    """Codes [..., 128 n] (any integer type) -> packed bytes of the 32-code group formats."""
    shape = codes.shape[:-1]
    f = (codes.to(torch.int16) & (2 ** bits - 1)).reshape(*shape, -1, 32)
    if bits == 8:
        return f.to(torch.uint8).reshape(*shape, -1)
    if bits == 4:
        f = f.reshape(*shape, -1, 2, 4)
        return ((f[..., 0, :] << 4) | f[..., 1, :]).to(torch.uint8).reshape(*shape, -1)
    f = f.reshape(*shape, -1, 8, 4)
    x0 = (f[..., 0, :] << 5) | (f[..., 1, :] << 2) | (f[..., 6, :] >> 1)
    x1 = (f[..., 2, :] << 5) | (f[..., 3, :] << 2) | (f[..., 7, :] >> 1)
    x2 = (f[..., 4, :] << 5) | (f[..., 5, :] << 2) | ((f[..., 7, :] & 1) << 1) | (f[..., 6, :] & 1)
    return torch.cat([x0, x1, x2], dim=-1).to(torch.uint8).reshape(*shape, -1)


def _unpack(packed, bits):
    """Packed bytes [..., n] -> int8 codes [..., 8 n / bits]."""
    shape = packed.shape[:-1]
    if bits == 8:
        return packed.view(torch.int8)
    if bits == 4:
        by = packed.reshape(*shape, -1, 1, 4)
        return torch.cat([by.view(torch.int8) >> 4, (by << 4).view(torch.int8) >> 4], dim=-2).reshape(*shape, -1)
    by = packed.reshape(*shape, -1, 3, 4)
    x0, x1, x2 = by[..., 0, :], by[..., 1, :], by[..., 2, :]
    f = torch.stack([x0 >> 5, (x0 >> 2) & 7, x1 >> 5, (x1 >> 2) & 7, x2 >> 5, (x2 >> 2) & 7,
                     ((x0 & 3) << 1) | (x2 & 1), ((x1 & 3) << 1) | ((x2 >> 1) & 1)], dim=-2)
    return ((f ^ 4).view(torch.int8) - 4).reshape(*shape, -1)


def _pages(gen, n_pages, d, page, bits):
    """Pages full of codes as quantizing to the clusters' ranges (three standard deviations to a side) leaves them."""
    out = torch.empty((n_pages, d // 128, page, 16 * bits), dtype=torch.uint8, device="cuda")
    at_once = max(1, (1 << 27) // (d * page))
    top = 2 ** (bits - 1)
    for i in range(0, n_pages, at_once):
        n = min(at_once, n_pages - i)
        codes = _normal(gen, n, d // 128, page, 128).mul_(2 ** bits / 6).sub_(0.5).round_().clamp_(-top, top - 1)
        out[i:i + n] = _pack(codes, bits)
    return out


def _batch(gen, case, st):
    """lens, page_table and the number of pages of B sequences."""
    B, page, per_seq = case["B"], case["page"], -(-case["most"] // case["page"])
    order = torch.randperm(B, generator=gen, device="cuda")
    st.lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")[order]
    used = -(-st.lens.long() // page)
    n_pages = int(used.sum()) + 3                                  # (a few that belong to nobody)
    mine = torch.arange(per_seq, device="cuda")[None, :] < used[:, None]
    ids = torch.randperm(n_pages, generator=gen, device="cuda")
    table = torch.full((B, per_seq), -1, dtype=torch.int64, device="cuda")
    table[mine] = ids[:int(used.sum())]
    gone = torch.tensor([[_hole(case, b, p) for p in range(per_seq)] for b in range(B)], device="cuda")[order]
    table[gone] = -1
    st.page_table = table.int()
    return n_pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 31)
    st = SimpleNamespace(case=case, cache=None, rotary=None, track=None, track_out=None, workspace=None)
    kind, hd = case["kind"], case["hd"]
    if kind in ("rope", "write"):
        st.freqs, st.amplitude = _frequencies(case)
        st.positions = _positions(gen, case["T"], case["far"])
    if kind == "rope":
        T, width = case["T"], case["heads"] * hd
        wide = _normal(gen, T, width + (width // 2 // hd * hd if case["packed"] else 0)).to(DTYPES[case["x"]])
        st.x = wide[:, :width]
        st.out = torch.zeros((T, width), dtype=DTYPES[case["out"]], device="cuda")
        return st
    H, bits, page = case["H"], case["bits"], case["page"]
    d = H * hd
    if kind == "write":
        T, width = case["T"], case["Hq"] * hd
        st.k_table, st.v_table = (_position_table(gen, H, hd, bits) for _ in range(2))
        n_pages = -(-T // page) + 3
        order = torch.randperm(n_pages, generator=gen, device="cuda")
        if T <= 64:                                                # a token each of T sequences, else a run of tokens
            st.slots = torch.randperm(n_pages * page, generator=gen, device="cuda")[:T].contiguous()
        else:
            st.slots = (order[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[5:T + 5].contiguous()
        st.k_pages, st.v_pages = (torch.zeros((n_pages, d // 128, page, 16 * bits), dtype=torch.uint8, device="cuda") for _ in range(2))
        if case["packed"]:
            qkv = _normal(gen, T, width + 2 * d).to(torch.bfloat16)
            st.q, st.k, st.v = qkv[:, :width], qkv[:, width:width + d], qkv[:, width + d:]
        else:
            st.q, st.k, st.v = (_normal(gen, T, n).to(torch.bfloat16) for n in (width, d, d))
        for x, table in ((st.k, st.k_table), (st.v, st.v_table)):  # (each channel as wide, and as far from zero, as its cluster)
            s, z = table[:, 2].view(torch.float32), table[:, 3].float()
            scale, shift = torch.empty_like(s), torch.empty_like(s)
            scale[table[:, 0].long()], shift[table[:, 0].long()] = s * (2 ** bits / 6), -z * s
            x.mul_(scale).add_(shift)
        st.q_out = torch.zeros((T, width), dtype=torch.bfloat16, device="cuda")
        return st
    B, most = case["B"], case["most"]
    n_pages = _batch(gen, case, st)
    if kind == "weights":
        Hq, n = case["Hq"], case["queries"]
        st.k_table = _position_table(gen, H, hd, bits)
        st.k_pages = _pages(gen, n_pages, d, page, bits)
        # queries for scores with a standard deviation around 1.5, sharper in some heads
        spread = st.k_table[:, 2].view(torch.float32).reshape(H, hd).mul(2 ** bits / 6).square().sum(1).sqrt()
        sharp = 1.5 * math.sqrt(hd) / spread[:, None] * torch.exp(0.5 * _normal(gen, H, Hq // H))
        st.q = (_normal(gen, B * n, Hq, hd) * sharp.reshape(Hq, 1)).to(torch.bfloat16).reshape(B * n, Hq * hd)
        st.positions = st.lens + 100                               # (of the newest token: some were evicted before)
        st.weights = torch.rand((B, H, most), generator=gen, device="cuda") * (4.0 / most)
        st.token_positions = torch.arange(most, dtype=torch.int32, device="cuda").expand(B, H, most).contiguous()
        st.lse = torch.empty((B * n, Hq), dtype=torch.float32, device="cuda")
        scores = _scores(st)                                       # what the attention of these queries left
        st.lse = torch.logsumexp(scores.double(), -1).permute(0, 3, 1, 2).reshape(B * n, Hq).float().contiguous()
        return st
    st.k_pages, st.v_pages = (torch.randint(0, 256, (n_pages, d // 128, page, 16 * bits), generator=gen, device="cuda", dtype=torch.uint8)
                              for _ in range(2))
    # a few tokens hold most of the weight, some have none at all
    w = torch.exp(2.5 * _normal(gen, B, H, most))
    st.weights = torch.where(torch.rand((B, H, most), generator=gen, device="cuda") < 0.03, 0.0, w)
    # what earlier evictions left is in no order, what came since is
    mixed = torch.rand((B, H, most), generator=gen, device="cuda")
    mixed[..., case["budget"] // 2:] = 2.0
    st.token_positions = torch.argsort(mixed, dim=-1, stable=True).int()
    st.weights_out = torch.zeros_like(st.weights)
    st.positions_out = torch.zeros_like(st.token_positions)
    st.lens_out = torch.zeros_like(st.lens)
    return st


# ---- one pass --------------------------------------------------------------------------------------------
def _rotary(st):
    """The framework's view of the frequencies, made once as a program does."""
    if st.rotary is None:
        import paper_2304_01089_amd as rp
        st.rotary = rp.Rotary(rotary_dim=st.case["rot"], freqs=st.freqs, amplitude=st.amplitude,
                              interleaved=st.case["style"] == "interleaved")
    return st.rotary


def _cache(st):
    """The framework's view of the pages, made once as a program does."""
    if st.cache is None:
        import paper_2304_01089_amd as rp
        c = st.case
        v_pages = getattr(st, "v_pages", st.k_pages)               # (the values of a cache whose weights alone are looked at)
        k_table = getattr(st, "k_table", None)
        st.cache = rp.PagedCache(n_heads=c["H"], head_dim=c["hd"], bits=c["bits"], page_size=c["page"], k_pages=st.k_pages,
                                 v_pages=v_pages, k_table=k_table, v_table=getattr(st, "v_table", k_table))
    return st.cache


def _turned(x, st):
    """Rows [T, n hd] rotated, fp32 (angles in 64 bits; two products and a sum, each rounded)."""
    c = st.case
    rot, hd, T = c["rot"], c["hd"], x.shape[0]
    angle = st.positions.double()[:, None] * st.freqs
    cos, sin = ((f(angle) * st.amplitude).float()[:, None] for f in (torch.cos, torch.sin))
    x = x.float().reshape(T, -1, hd)
    if c["style"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).reshape(T, -1, rot)
    return torch.cat([turned, x[..., rot:]], dim=-1).reshape(T, -1)


def _scores(st):
    """[B, H, Hq / H, queries, tokens] of every query and the tokens that it sees (else -inf), fp32."""
    c = st.case
    B, H, Hq, hd, n, page, bits = c["B"], c["H"], c["Hq"], c["hd"], c["queries"], c["page"], c["bits"]
    ids, table = st.page_table.long(), st.k_table
    tokens = ids.shape[1] * page
    rows = st.k_pages[ids.clamp(0, st.k_pages.shape[0] - 1)].transpose(2, 3).reshape(B, tokens, -1)
    k = (_unpack(rows, bits).float() - table[:, 3].float()) * table[:, 2].view(torch.float32)
    k = k.reshape(B, tokens, H, hd).transpose(1, 2).contiguous()
    q = st.q.float().reshape(B, n, H, Hq // H, hd).permute(0, 2, 3, 1, 4).reshape(B, H, Hq // H * n, hd)
    order = (table[:, 0].long().reshape(H, 1, hd) - hd * torch.arange(H, device="cuda").reshape(H, 1, 1)).expand_as(q)
    scores = q.gather(-1, order).matmul(k.transpose(-1, -2).contiguous()).reshape(B, H, Hq // H, n, tokens) / math.sqrt(hd)
    here = ((ids >= 0) & (ids < st.k_pages.shape[0])).repeat_interleave(page, dim=1)[:, None]
    last = st.lens[:, None] - (n - 1) + torch.arange(n, device="cuda")
    here = here & (torch.arange(tokens, device="cuda") < last[..., None])
    return torch.where(here[:, None, None], scores, float("-inf"))


def _sources(weights, positions, lens, there, budget, first, recent):
    """Where every token of the result comes from [B, H, most], and the new lengths."""
    t = torch.arange(weights.shape[-1], device="cuda")
    mine = (t < lens[:, None])[:, None]
    newest = torch.where(mine, positions, -2 ** 31).amax(-1, keepdim=True)
    bits = (weights + 0.0).view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -1 - (bits & 0x7fffffff))
    key = torch.where(weights.isnan(), 2 ** 40, key)
    key = torch.where((positions < first) | (positions > newest - recent), 2 ** 41, key)
    key = torch.where(mine, key, -2 ** 40)
    ranked = torch.argsort(key, dim=-1, descending=True, stable=True)[..., :budget]
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, ranked, True)
    hole, moved = ~kept & (t < budget), kept & (t >= budget)
    from_behind = torch.argsort((~moved).int(), dim=-1, stable=True)
    rank = (hole.cumsum(-1) - 1).clamp_min(0)
    cut = ((lens > budget) & there)[:, None, None]
    return torch.where(hole & cut, from_behind.gather(-1, rank), t), torch.where(cut[:, 0, 0], budget, lens)


def _by_head(pages, H, hd):
    """Pages as [pages, heads, pieces, tokens, bytes] (narrow heads: [pages, blocks, heads of a block, tokens, bytes]), a view."""
    n, blocks, page, row = pages.shape
    if hd > 128:
        return pages.view(n, H, hd // 128, page, row)
    return pages.view(n, blocks, page, 128 // hd, row * hd // 128).permute(0, 1, 3, 2, 4)


def _head_at(h, hd):
    """Indices of heads in what _by_head gives, between the page's and the token's."""
    return (h, slice(None)) if hd > 128 else (h // (128 // hd), h % (128 // hd))


def run(st):
    case = st.case
    kind, hd = case["kind"], case["hd"]
    if own:
        import paper_2304_01089_amd as rp
        if kind == "rope":
            rp.rope(_rotary(st), st.x, st.positions, hd, out=st.out)
            return dict(out=st.out)
        cache = _cache(st)
        if kind == "write":
            rp.rope_quant_paged(cache, _rotary(st), st.q, st.k, st.v, st.positions, st.slots, q_out=st.q_out)
            return dict(q=st.q_out, k_pages=st.k_pages, v_pages=st.v_pages)
        if st.track is None:
            st.track = rp.CacheTrack(weights=st.weights, positions=st.token_positions)
        if kind == "weights":
            rp.attend_weights_paged(cache, st.q, st.page_table, st.lens, st.lse, st.track, positions=st.positions,
                                    queries=case["queries"], fresh=1 if case["fresh"] == "one" else case["most"])
            return dict(weights=st.weights, positions=st.token_positions)
        if st.workspace is None:
            st.track_out = rp.CacheTrack(weights=st.weights_out, positions=st.positions_out)
            st.workspace = rp.evict_paged_workspace(cache, case["B"], case["most"], case["budget"])
        rp.evict_paged(cache, st.page_table, st.lens, st.track, case["budget"], first=case["first"], recent=case["recent"],
                       out=st.track_out, lens_out=st.lens_out, workspace=st.workspace)
        return dict(k_pages=st.k_pages, v_pages=st.v_pages, weights=st.weights_out, positions=st.positions_out, lens=st.lens_out)
    if kind == "rope":
        st.out.copy_(_turned(st.x, st))
        return dict(out=st.out)
    if kind == "write":
        bits, page, top = case["bits"], case["page"], 2 ** (case["bits"] - 1)
        st.q_out.copy_(_turned(st.q, st))
        for x, table, pages in ((_turned(st.k, st), st.k_table, st.k_pages), (st.v.float(), st.v_table, st.v_pages)):
            r = torch.round(x[:, table[:, 0].long()] * table[:, 1].view(torch.float32))
            codes = torch.clamp(r + table[:, 3].float(), -top, top - 1)
            pages[st.slots // page, :, st.slots % page] = _pack(codes, bits).reshape(case["T"], -1, 16 * bits)
        return dict(q=st.q_out, k_pages=st.k_pages, v_pages=st.v_pages)
    if kind == "weights":
        B, H, n, most = case["B"], case["H"], case["queries"], case["most"]
        lse = st.lse.reshape(B, n, H, -1).permute(0, 2, 3, 1)[..., None]
        scores = _scores(st)[..., :most]
        got = torch.where(scores == float("-inf"), 0.0, torch.exp(scores - lse)).sum((2, 3))
        t = torch.arange(most, device="cuda")
        mine = (t < st.lens[:, None])[:, None]
        starts = mine & (t >= st.lens[:, None] - (1 if case["fresh"] == "one" else most))[:, None]
        st.weights.copy_(torch.where(starts, got, torch.where(mine, st.weights + got, st.weights)))
        at = st.positions[:, None] - (st.lens[:, None] - 1 - t)
        st.token_positions.copy_(torch.where(starts, at[:, None].int(), st.token_positions))
        return dict(weights=st.weights, positions=st.token_positions)
    page, H = case["page"], case["H"]
    ids = st.page_table.long()
    used = torch.arange(ids.shape[1], device="cuda") * page < st.lens[:, None]
    there = (((ids >= 0) & (ids < st.k_pages.shape[0])) | ~used).all(-1)
    src, lens = _sources(st.weights, st.token_positions, st.lens, there, case["budget"], case["first"], case["recent"])
    t = torch.arange(case["most"], device="cuda")
    b, h, to = torch.nonzero((src != t), as_tuple=True)
    fro = src[b, h, to]
    for pages in (st.k_pages, st.v_pages):
        view, at = _by_head(pages, H, hd), _head_at(h, hd)
        view[(ids[b, to // page],) + at + (to % page,)] = view[(ids[b, fro // page],) + at + (fro % page,)]
    mine = (t < lens[:, None])[:, None]
    st.weights_out.copy_(torch.where(mine, st.weights.gather(-1, src), st.weights_out))
    st.positions_out.copy_(torch.where(mine, st.token_positions.gather(-1, src), st.positions_out))
    st.lens_out.copy_(lens)
    return dict(k_pages=st.k_pages, v_pages=st.v_pages, weights=st.weights_out, positions=st.positions_out, lens=st.lens_out)


# ---- what a pass cannot do without -------------------------------------------------------------------------
def work(case):
    kind, hd = case["kind"], case["hd"]
    if kind == "rope":
        size = {"bf16": 2, "f32": 4}
        values = case["T"] * case["heads"] * hd
        return dict(bytes=values * (size[case["x"]] + size[case["out"]]) + 4 * case["T"] + 4 * case["rot"],
                    flops=3 * case["T"] * case["heads"] * case["rot"])
    H, bits = case["H"], case["bits"]
    d = H * hd
    if kind == "write":
        T, q = case["T"], case["Hq"] * hd
        return dict(bytes=T * (4 * q + 2 * d * (2 + bits / 8) + 12) + 32 * d + 4 * case["rot"],
                    flops=3 * T * (case["Hq"] + H) * case["rot"])
    lens = _lengths(case)
    if kind == "weights":
        tokens = 0
        for b, n in enumerate(lens):
            tokens += sum(min(case["page"], n - p * case["page"]) for p in range(-(-n // case["page"])) if not _hole(case, b, p))
        asked = case["B"] * case["queries"] * case["Hq"] * (2 * hd + 4)
        return dict(bytes=tokens * d * bits / 8 + sum(lens) * H * 8 + asked + 16 * d, flops=2 * case["Hq"] * hd * case["queries"] * tokens)
    budget, read, moved = case["budget"], 0, 0
    for b, n in enumerate(lens):
        gone = any(_hole(case, b, p) for p in range(-(-n // case["page"])))
        read += 8 * (n + min(n, n if gone else budget))
        moved += 0 if gone or n <= budget else budget * (n - budget) / n     # (kept tokens lie anywhere)
    return dict(bytes=H * (read + moved * 4 * hd * bits / 8) + 8 * case["B"], flops=0)


# ---- the same in 64 bits ------------------------------------------------------------------------------------
def _codes64(packed, bits):
    """Codes as int64 [..., 32] of packed groups [..., 4 bits bytes], field by field as the formats are written down."""
    b = packed.long()
    if bits == 8:
        f = b
    elif bits == 4:
        f = torch.stack([(b[..., 4 * (j // 8) + j % 4] >> (4 if j % 8 < 4 else 0)) & 15 for j in range(32)], dim=-1)
    else:
        f = []
        for j in range(32):
            e, i = j // 4, j % 4
            if e < 6:
                f.append((b[..., 4 * (e // 2) + i] >> (5 if e % 2 == 0 else 2)) & 7)
            else:
                f.append((b[..., 4 * (e - 6) + i] & 3) * 2 + ((b[..., 8 + i] >> (e - 6)) & 1))
        f = torch.stack(f, dim=-1)
    return torch.where(f >= 2 ** (bits - 1), f - 2 ** bits, f)


def _rotate64(x, st):
    """Pair after pair, in complex numbers."""
    c = st.case
    y = x.double().reshape(x.shape[0], -1, c["hd"]).clone()
    for j in range(c["rot"] // 2):
        a, b = (j, j + c["rot"] // 2) if c["style"] == "half" else (2 * j, 2 * j + 1)
        turn = torch.polar(torch.full_like(st.freqs[0], st.amplitude), st.positions.double() * st.freqs[j])
        z = torch.complex(y[..., a], y[..., b]) * turn[:, None]
        y[..., a], y[..., b] = z.real, z.imag
    return y.reshape(x.shape[0], -1)


def exact(case, seed):
    st = prepare(case, seed)
    kind, hd = case["kind"], case["hd"]
    if kind == "rope":
        return dict(out=_rotate64(st.x, st))
    if kind == "write":
        # (codes are whole numbers that depend on how the rotated value is rounded: that is part of the definition, not of 64 bits)
        return dict(q=_rotate64(st.q, st), k_pages=None, v_pages=None)
    H, bits, page, B, most = case["H"], case["bits"], case["page"], case["B"], case["most"]
    if kind == "weights":
        n, Hq = case["queries"], case["Hq"]
        share = Hq // H
        out = st.weights.double()
        s, z = st.k_table[:, 2].view(torch.float32).double(), st.k_table[:, 3].double()
        by_channel = torch.empty(H * hd, dtype=torch.long, device="cuda")
        by_channel[st.k_table[:, 0].long()] = torch.arange(H * hd, device="cuda")
        for b in range(B):
            length = int(st.lens[b])
            t = torch.arange(length, device="cuda")
            start = max(0, length - (1 if case["fresh"] == "one" else most))
            out[b, :, start:length] = 0.0
            ids = st.page_table[b].long()[t // page]
            t, ids = t[ids >= 0], ids[ids >= 0]
            for lo in range(0, len(t), 2048):
                at, pid = t[lo:lo + 2048], ids[lo:lo + 2048]
                rows = st.k_pages[pid, :, at % page].reshape(len(at), -1, 4 * bits)
                k = (s * (_codes64(rows, bits).reshape(len(at), -1).double() - z))[:, by_channel].reshape(-1, H, hd)
                for i in range(n):
                    q = st.q[b * n + i].double().reshape(H, share, hd)
                    a = torch.stack([(k * q[:, g]).sum(-1) for g in range(share)], dim=-1) / math.sqrt(hd)      # [tokens, H, share]
                    p = torch.exp(a - st.lse[b * n + i].double().reshape(H, share)).sum(-1)
                    out[b][:, at] += torch.where((at < length - (n - 1 - i))[:, None], p, 0.0).T
        return dict(weights=out, positions=None)
    # whole rows that move: head after head, by sorting
    out = np.zeros((B, H, most))
    w, pos, lens, table = (x.cpu().numpy() for x in (st.weights, st.token_positions, st.lens, st.page_table))
    for b in range(B):
        n = int(lens[b])
        if n == 0:
            continue
        stays = n <= case["budget"] or bool((table[b, :-(-n // page)] < 0).any())
        for h in range(H):
            a = w[b, h, :n].astype(np.float64)
            if stays:
                out[b, h, :n] = a
                continue
            p = pos[b, h, :n].astype(np.int64)
            safe = (p < case["first"]) | (p > p.max() - case["recent"])
            best = np.lexsort((np.arange(n), -a, ~safe))[:case["budget"]]
            keep = np.zeros(n, bool)
            keep[best] = True
            at = np.arange(n)
            a[at[:case["budget"]][~keep[:case["budget"]]]] = a[at[case["budget"]:][keep[case["budget"]:]]]
            out[b, h, :case["budget"]] = a[:case["budget"]]
    return dict(k_pages=None, v_pages=None, weights=torch.from_numpy(out), positions=None, lens=None)
