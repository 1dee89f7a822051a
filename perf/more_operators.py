"""Timed cases of the operators of long contexts on a compressed cache: rotary positions, keys and values in 4 bits, attention over
them, and the eviction of the tokens that got least of it.

  rotary       heads of rows turned by their positions: half or interleaved pairs, the whole head or its first part, frequencies
               stretched for long contexts; `inverse` is the gradient
  append       new keys and values rounded to 4 bits (32 values share a power of two) and stored in a paged cache, then read back
  attention    rows of queries over the cached tokens of their request; with `weight` every token's probability is added to its weight
  evict        a request's cache cut to a budget of tokens a head: the first, the newest and those of largest weight stay

With `own` false each is computed in its plain form (elementary torch operations, fp32 inside, angles in 64 bits), with `own` true by
the library's entry points."""
import math
import random

import torch

own = False

DEV = "cuda"
RMS_EPS, THETA = 1e-6, 1e4
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)          # the magnitudes of a 4-bit value


def _rotary(name, n, heads, hd, rot, dtype, interleaved=False, inverse=False, factor=1.0, original=0, far=4096, pad=0):
    return dict(name=name, op="rotary", n=n, heads=heads, hd=hd, rot=rot, dtype=dtype, interleaved=interleaved, inverse=inverse, factor=factor,
                original=original, far=far, pad=pad)


def _append(name, n, hkv, hd, dtype, per_head=False, pad=0.0):
    return dict(name=name, op="append", n=n, hkv=hkv, hd=hd, dtype=dtype, block=16, per_head=per_head, pad=pad)


def _attention(name, reqs, lo, hi, hq, hkv, hd, dtype="bf16", rows_lo=1, rows_hi=1, weight=False, per_head=False, block=16, lens=1):
    return dict(name=name, op="attention", reqs=reqs, lo=lo, hi=hi, hq=hq, hkv=hkv, hd=hd, dtype=dtype, rows_lo=rows_lo, rows_hi=rows_hi, weight=weight,
                per_head=per_head, block=block, lens=lens)


def _evict(name, reqs, lo, hi, budget, hkv, hd, sinks, recent, spread=0.0, block=16, lens=1):
    return dict(name=name, op="evict", reqs=reqs, lo=lo, hi=hi, budget=budget, hkv=hkv, hd=hd, sinks=sinks, recent=recent, spread=spread, block=block,
                lens=lens)


def listed():
    return [
        # queries and keys of the new tokens of a decode-only iteration of the edge configuration, read from the rows of the joint product
        _rotary("rotary_decode_edge", 32, 40, 64, 64, "bf16", far=2048, pad=512),
        # all rows of the fine-tune-heavy iteration; interleaved pairs in half of each head, a context four times as long as the trained one
        _rotary("rotary_7b_part_long", 66576, 64, 128, 64, "bf16", interleaved=True, factor=4.0, original=8192, far=32768),
        # gradient of queries and keys kept in fp32, ragged number of rows
        _rotary("rotary_grad_fp32", 12289, 40, 128, 128, "fp32", inverse=True, factor=8.0, original=4096, far=16384),
        # the new tokens of a decode batch, every head at a place of its own (heads of different budgets), two rows not to be stored
        _append("append_decode_7b", 64, 32, 128, "bf16", per_head=True, pad=0.03),
        # prompts of grouped heads on their way into the cache
        _append("append_prefill_gqa", 16384, 8, 128, "bf16"),
        # the decode rows of the fp32 configuration: one small launch
        _attention("attention_tiny_fp32", 4, 32, 128, 4, 4, 64, "fp32"),
        # the decode batch of the edge configuration, weights kept for eviction
        _attention("attention_decode_edge", 32, 256, 2048, 32, 8, 64, weight=True),
        # half of the requests of the decode-heavy configuration: the stream of the cache sets the time
        _attention("attention_decode_7b", 128, 2048, 8192, 32, 32, 128),
        # one request at the end of a long document, grouped heads
        _attention("attention_long_one", 1, 131001, 131001, 32, 8, 128),
        # pieces of prompts behind long cached contexts, ragged, weights kept
        _attention("attention_pieces_gqa", 6, 2000, 8000, 32, 8, 128, rows_lo=37, rows_hi=256, weight=True),
        # the edge batch a little over its budget: few tokens go, all latency
        _evict("evict_step_edge", 32, 1025, 1088, 1024, 8, 64, 4, 128),
        # long documents cut to half, budgets by the heads' norms
        _evict("evict_long_gqa", 8, 20000, 32768, 12000, 8, 128, 4, 512, spread=0.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "append", "attention", "attention", "attention", "evict"))
    hd = rng.choice((64, 128))
    hkv = rng.choice((4, 8, 32))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    if op == "rotary":
        heads = _log_int(rng, 4, 64)
        factor = rng.choice((1.0, 2.0, 8.0))
        n = _log_int(rng, 1, 66576 * 64 * 128 // (heads * hd) // (2 if dtype == "fp32" else 1) // 4)
        c = _rotary("", n, heads, hd, rng.choice((hd, hd // 2, 16, 24)), dtype, rng.random() < 0.5, rng.random() < 0.4, factor,
                    rng.choice((0, 4096)), _log_int(rng, 1000, 200000), 8 * rng.randrange(0, 40))
    elif op == "append":
        c = _append("", _log_int(rng, 1, 16384 * 8 // hkv), hkv, hd, dtype, rng.random() < 0.4, rng.choice((0.0, 0.05)))
    elif op == "attention":
        group = rng.choice((1, 2, 4, 8))
        block = rng.choice((8, 16, 16, 64))
        lens = rng.randrange(1, 1 << 20)
        if rng.random() < 0.35:
            group = min(group, 64 // hkv)
            hi = _log_int(rng, 40, 8000)
            rows = _log_int(rng, 2, 256)
            reqs = _log_int(rng, 1, max(1, min(8, 6 * 8000 * 256 * 32 * 128 // ((hi + rows) * rows * hkv * group * hd))))
            c = _attention("", reqs, hi // 3, hi, hkv * group, hkv, hd, dtype, max(1, rows // 4), rows, rng.random() < 0.5, False, block, lens)
        else:
            hi = _log_int(rng, 40, 60000)
            reqs = _log_int(rng, 1, max(1, min(128, 64 * 5000 * 32 * 128 // (hi * hkv * hd))))
            c = _attention("", reqs, hi // 4, hi, hkv * group, hkv, hd, dtype, 1, 1, rng.random() < 0.4, rng.random() < 0.4, block, lens)
    else:
        hi = _log_int(rng, 100, 32768)
        lo = hi - _log_int(rng, 1, hi // 2)
        reqs = _log_int(rng, 1, max(1, min(32, 8 * 32768 * 8 // (hi * hkv))))
        c = _evict("", reqs, lo, hi, _log_int(rng, max(1, hi // 4), hi), hkv, hd, rng.choice((0, 4, 17)), rng.choice((0, 32, hi // 8)),
                   rng.choice((0.0, 0.3)), rng.choice((8, 16, 64)), rng.randrange(1, 1 << 20))
    del c["name"]
    return c


def _lengths(case):
    """Cached tokens (of every head, where they differ) and new rows of each request: a function of the case alone."""
    rng = random.Random(case["lens"])
    tokens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["reqs"])]
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in tokens] if case["op"] == "attention" else [0] * len(tokens)
    heads = [[rng.randint(max(1, t // 2), t) for _ in range(case["hkv"])] if case.get("per_head") else [t] * case["hkv"] for t in tokens]
    return heads, rows


def _budgets(case):
    rng = random.Random(case["lens"] + 1)
    return [[max(1, round(case["budget"] * (1.0 + case["spread"] * rng.uniform(-1.0, 1.0)))) for _ in range(case["hkv"])] for _ in range(case["reqs"])]


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class _Handle:
    def __init__(self, hq, hkv, hd, bf16):
        from paper_2510_03283_amd import binding as B
        self.B = B
        self.h = B.mace_create(4096, hq, hkv, hd, 64, 64, RMS_EPS, THETA, B.MACE_BF16 if bf16 else B.MACE_F32)

    def __del__(self):
        self.B.mace_destroy(self.h)


class _State:
    pass


def _frequencies(case):
    """Frequencies of the pairs in 64 bits: those that turn less than once over the trained context are divided by the factor, those that turn
    more than 32 times stay, between the two a straight line; without a trained length all are divided."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64)
    f = THETA ** (-2.0 * i / case["rot"])
    keep = ((case["original"] * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0) if case["original"] else torch.zeros_like(f)
    return f * (keep + (1.0 - keep) / case["factor"])


def _pool(s, case, gen, blocks):
    """A pool of cache blocks as earlier steps filled it: codes, and scales of values of spread about 1."""
    shape = (blocks, case["hkv"], case["block"])
    codes = lambda: torch.randint(0, 256, (*shape, case["hd"] // 2), generator=gen, device=DEV, dtype=torch.uint8)
    scales = lambda: torch.randint(124, 127, (*shape, case["hd"] // 32), generator=gen, device=DEV, dtype=torch.uint8)
    s.k, s.v, s.k_scale, s.v_scale = codes(), codes(), scales(), scales()
    return shape


def _tables(s, case, gen, tokens):
    """Block tables of requests whose blocks lie anywhere in the pool, which is an eighth larger than they need."""
    need = [-(-t // case["block"]) for t in tokens]
    blocks = sum(need) + max(1, sum(need) // 8)
    order = torch.randperm(blocks, generator=gen, device=DEV).int()
    s.tables = torch.full((len(need), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for r, m in enumerate(need):
        s.tables[r, :m] = order[at:at + m]
        at += m
    return blocks


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = _State()
    s.case = case
    dtype = DTYPES[case.get("dtype", "bf16")]
    if own:
        hq, hkv = case.get("hq", case.get("hkv", 4)), case.get("hkv", 4)
        s.handle = _Handle(hq, hkv, case["hd"], dtype == torch.bfloat16)
    work_bytes = 0
    if case["op"] == "rotary":
        n, d = case["n"], case["heads"] * case["hd"]
        s.x = torch.randn((n, d + case["pad"]), generator=gen, device=DEV).to(dtype)
        s.out = torch.empty((n, d), dtype=dtype, device=DEV)
        s.positions = torch.randint(0, case["far"], (n,), generator=gen, device=DEV, dtype=torch.int32)
        s.frequencies = _frequencies(case).to(DEV)
        s.magnitude = 0.1 * math.log(case["factor"]) + 1.0
    elif case["op"] == "append":
        n, hkv, hd, block = case["n"], case["hkv"], case["hd"], case["block"]
        # groups of very different size, as keys have them; a few zeros
        spread = torch.exp(torch.randn((2, n, hkv * hd // 32, 1), generator=gen, device=DEV))
        x = torch.randn((2, n, hkv * hd // 32, 32), generator=gen, device=DEV) * spread
        x[:, torch.rand(n, generator=gen, device=DEV) < 0.01] = 0.0
        s.k_new, s.v_new = x.view(2, n, hkv * hd).to(dtype)
        blocks = -(-(n + 8) // block) + 4
        slots = lambda: torch.randperm(blocks * block, generator=gen, device=DEV)[:n].int()
        s.slots = torch.stack([slots() for _ in range(hkv)], dim=1) if case["per_head"] else slots()
        if case["pad"]:
            s.slots[torch.rand(n, generator=gen, device=DEV) < case["pad"]] = -1
        _pool(s, case, gen, blocks)
        s.k_out, s.v_out = torch.empty_like(s.k_new), torch.empty_like(s.v_new)
    elif case["op"] == "attention":
        heads, rows = _lengths(case)
        s.max_context, s.max_rows, s.n_rows = max(map(max, heads)), max(rows), sum(rows)
        shape = _pool(s, case, gen, _tables(s, case, gen, [max(t) + n for t, n in zip(heads, rows)]))
        s.weight = torch.rand(shape, generator=gen, device=DEV) if case["weight"] else None
        s.lens = _int(heads) if case["per_head"] else _int([t[0] for t in heads])
        s.offsets = _int([sum(rows[:i]) for i in range(len(rows) + 1)]) if s.max_rows > 1 else None
        # some rows attend sharply, some widely
        s.q = (torch.randn((s.n_rows, case["hq"] * case["hd"]), generator=gen, device=DEV) * (0.5 + 2.5 * torch.rand((s.n_rows, 1), generator=gen, device=DEV))).to(dtype)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty((s.n_rows, case["hq"]), dtype=torch.float32, device=DEV)
        s.scale = case["hd"] ** -0.5
        if own:
            work_bytes = s.handle.B.mace_kv4_attention_workspace_bytes(s.handle.h, case["reqs"], s.max_rows, s.max_context)
    else:
        heads, _ = _lengths(case)
        shape = _pool(s, case, gen, _tables(s, case, gen, [t[0] for t in heads]))
        s.max_context = max(map(max, heads))
        s.lens, s.budgets = _int([t[0] for t in heads]), _int(_budgets(case))
        s.seen = 2 * s.lens                                    # tokens of the request so far; half of them are gone
        # weights fall off steeply, some tokens never got any; positions: the newest in order at the end, the others anywhere before
        weight = torch.rand(shape, generator=gen, device=DEV) ** 6
        weight[torch.rand(shape, generator=gen, device=DEV) < 0.05] = 0.0
        position = torch.zeros(shape, dtype=torch.int32, device=DEV)
        tail = max(case["recent"], case["lo"] // 16)
        for r, t in enumerate(heads):
            t = t[0]
            old = torch.rand((case["hkv"], 2 * t - tail), generator=gen, device=DEV).argsort(dim=1)[:, :t - tail]
            new = torch.arange(2 * t - tail, 2 * t, device=DEV).expand(case["hkv"], tail)
            block, off = _places(s, r, t)
            position[block, :, off] = torch.cat([old, new], dim=1).T.int()
        s.book0 = torch.stack([weight.view(torch.int32), position])
        s.book = s.book0.clone()
        s.weight, s.position = s.book[0].view(torch.float32), s.book[1]
        s.new_lens = torch.empty_like(s.budgets)
        if own:
            work_bytes = s.handle.B.mace_kv4_evict_workspace_bytes(s.handle.h, case["reqs"], s.max_context)
    if own:
        s.work = torch.empty(max(work_bytes, 256), dtype=torch.uint8, device=DEV)
        if hasattr(s, "k"):
            s.cache = s.handle.B.kv4_cache_struct(s.k, s.v, s.k_scale, s.v_scale, getattr(s, "weight", None), getattr(s, "position", None))
    return s


def _places(s, r, t):
    """(block, place in it) of the first t tokens of request r."""
    i = torch.arange(t, device=DEV)
    return s.tables[r].long()[i // s.case["block"]], i % s.case["block"]


# ---- plain forms ----

def _plain_rotary(s):
    case = s.case
    n, heads, hd, rot = case["n"], case["heads"], case["hd"], case["rot"]
    angle = s.positions.double()[:, None] * s.frequencies
    cos, sin = (s.magnitude * angle.cos()).float()[:, None], (s.magnitude * angle.sin()).float()[:, None]
    if case["inverse"]:
        sin = -sin
    x = s.x[:, :heads * hd].reshape(n, heads, hd)
    pairs = x[..., :rot].float()
    a, b = (pairs[..., 0::2], pairs[..., 1::2]) if case["interleaved"] else (pairs[..., :rot // 2], pairs[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).flatten(2) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return {"out": torch.cat([turned.to(x.dtype), x[..., rot:]], dim=-1).view(n, heads * hd)}


def _power(e):
    """2^e in fp32, from its bits (a function of the device may be off by a step, and values next to a border go by it)."""
    return (e.int() + 127 << 23).view(torch.float32)


def _rounded(x):
    """Rows [..., hd] -> bytes of two codes each, the first in the low half, and a scale byte for every 32 values."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(dim=-1, keepdim=True)
    half, exponent = torch.frexp(top)                                   # top = half 2^exponent, half in [1/2, 1)
    e = torch.where(top == 0, -124, (exponent - 3 + (half > 0.875)).clamp(-124, 125))
    y = x.abs() * _power(-e)
    code = (y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
    code = (code | torch.signbit(x).byte() << 3).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).byte()[..., 0]


def _values(codes, scales):
    """fp32 values of stored rows."""
    table = torch.tensor([[sign * g for sign in (1.0, -1.0) for g in GRID]], device=codes.device)[0]
    byte = torch.arange(256, device=codes.device)
    pairs = torch.stack([table[byte & 15], table[byte >> 4]], dim=1)
    x = pairs[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    return (x * _power(scales.int() - 127)[..., None]).flatten(-2)


def _plain_append(s):
    case = s.case
    n, hkv, hd, block = case["n"], case["hkv"], case["hd"], case["block"]
    slots = s.slots if case["per_head"] else s.slots[:, None].expand(n, hkv)
    there = slots >= 0
    row, head = there.nonzero(as_tuple=True)
    slot = slots[row, head].long()
    out = {}
    for name, new, codes, scales, to in (("k", s.k_new, s.k, s.k_scale, s.k_out), ("v", s.v_new, s.v, s.v_scale, s.v_out)):
        c, e = _rounded(new.view(n, hkv, hd))
        codes[slot // block, head, slot % block], scales[slot // block, head, slot % block] = c[row, head], e[row, head]
        to.zero_()
        to.view(n, hkv, hd)[row, head] = _values(codes[slot // block, head, slot % block], scales[slot // block, head, slot % block]).to(to.dtype)
        out[name] = to
    return out


def _cached(s, codes, scales):
    """fp32 rows [requests, kv heads, tokens, hd] of all blocks of the tables (those that a request lacks: any)."""
    t = s.tables.clamp(min=0).long()
    return _values(codes[t].transpose(1, 2).flatten(2, 3), scales[t].transpose(1, 2).flatten(2, 3))


def _plain_attention(s):
    case = s.case
    reqs, hkv, hd, group, most = case["reqs"], case["hkv"], case["hd"], case["hq"] // case["hkv"], s.max_rows
    k = _cached(s, s.k, s.k_scale)
    tokens = k.shape[2]
    offsets = s.offsets if s.offsets is not None else torch.arange(reqs + 1, device=DEV)
    i = torch.arange(most, device=DEV)
    row = offsets[:-1, None] + i                                        # [requests, most]
    real = row < offsets[1:, None]
    q = s.q.float()[torch.where(real, row, 0)].view(reqs, most, hkv, group, hd).permute(0, 2, 3, 1, 4).reshape(reqs, hkv, group * most, hd)
    lens = s.lens if case["per_head"] else s.lens[:, None].expand(reqs, hkv)
    seen = torch.arange(tokens, device=DEV) <= lens[:, :, None, None] + i[:, None]         # [requests, hkv, most, tokens]
    logits = (q @ k.transpose(-1, -2)).view(reqs, hkv, group, most, tokens) * s.scale
    del k
    logits = logits.masked_fill(~seen[:, :, None], -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    p = (logits - top).exp()
    total = p.sum(dim=-1, keepdim=True)
    p /= total
    lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(reqs, most, case["hq"])
    if case["weight"]:
        got = (p * real[:, None, None, :, None]).sum(dim=(2, 3))                           # [requests, hkv, tokens]
        got = got.view(reqs, hkv, -1, case["block"]).transpose(1, 2)
        there = s.tables >= 0
        s.weight[s.tables[there].long()] += got[there]
    v = _cached(s, s.v, s.v_scale)
    o = (p.view(reqs, hkv, group * most, tokens) @ v).view(reqs, hkv, group, most, hd).permute(0, 3, 1, 2, 4).reshape(reqs, most, case["hq"] * hd)
    out = {"out": o[real].to(s.q.dtype), "lse": lse[real]}
    if case["weight"]:
        out["weight"] = s.weight
    return out


def _plain_evict(s):
    case = s.case
    reqs, hkv, block = case["reqs"], case["hkv"], case["block"]
    s.book.copy_(s.book0)                                      # weights and positions as the steps before left them
    most = s.max_context
    i = torch.arange(most, device=DEV)
    blk = s.tables.clamp(min=0).long()[:, i // block][:, None].expand(reqs, hkv, most)
    head, off = torch.arange(hkv, device=DEV)[None, :, None].expand_as(blk), (i % block).expand_as(blk)
    weight, position = s.weight[blk, head, off], s.position[blk, head, off].long()
    key = torch.where(weight > 0, weight, 0.0).view(torch.int32).long()
    key = torch.where(position >= s.seen[:, None, None] - case["recent"], (1 << 31) + position, key)
    key = torch.where(position < case["sinks"], (3 << 30) + (1 << 30) - 1 - position, key)
    held = i < s.lens[:, None, None]
    order = torch.where(held, (key << 31) + (2**31 - 1 - i), -1 - i).argsort(dim=2, descending=True)
    new = torch.minimum(s.lens[:, None], s.budgets)
    keep = torch.zeros_like(held.expand(reqs, hkv, most)).scatter(2, order, i < new[:, :, None])
    front = i < new[:, :, None]
    hole, moved = front & ~keep, keep & ~front
    r, h, to = hole.nonzero(as_tuple=True)                     # both in order: the i-th hole gets the i-th of the moved
    _, _, frm = moved.nonzero(as_tuple=True)
    place = lambda t: (blk[r, h, t], h, off[r, h, t])
    for x in (s.k, s.v, s.k_scale, s.v_scale, s.weight, s.position):
        x[place(to)] = x[place(frm)]
    s.new_lens.copy_(new)
    return _evicted(s)


def _evicted(s):
    # rows are moved, not computed: their bytes, as they lie in the pool
    return {"lens": s.new_lens, "k": s.k, "v": s.v, "k_scale": s.k_scale, "v_scale": s.v_scale, "weight": s.weight, "position": s.position}


def run(s):
    case = s.case
    op = case["op"]
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "attention": _plain_attention, "evict": _plain_evict}[op](s)
    B, h = s.handle.B, s.handle.h
    if op == "rotary":
        B.mace_rotary(h, s.x, s.positions, s.frequencies, s.out, case["heads"], interleaved=case["interleaved"], magnitude=s.magnitude, inverse=case["inverse"])
        return {"out": s.out}
    if op == "append":
        B.mace_kv4_append(h, s.cache, s.k_new, s.v_new, s.slots)
        B.mace_kv4_gather(h, s.cache, s.slots, s.k_out, s.v_out)
        return {"k": s.k_out, "v": s.v_out}
    if op == "attention":
        B.mace_kv4_attention(h, s.cache, s.q, s.tables, s.lens, s.out, s.work, s.max_context, q_offsets=s.offsets, max_rows=s.max_rows, lse=s.lse,
                             scale=s.scale, add_weight=case["weight"])
        out = {"out": s.out, "lse": s.lse}
        if case["weight"]:
            out["weight"] = s.weight
        return out
    s.book.copy_(s.book0)                                      # weights and positions as the steps before left them
    B.mace_kv4_evict(h, s.cache, s.tables, s.lens, s.seen, s.budgets, s.new_lens, s.work, s.max_context, n_sink=case["sinks"], n_recent=case["recent"])
    return _evicted(s)


def _size(case):
    return 4 if case.get("dtype") == "fp32" else 2


def work(case):
    op = case["op"]
    if op == "rotary":
        values = case["n"] * case["heads"] * case["hd"]
        return {"bytes": 2 * values * _size(case) + 4 * case["n"] + 4 * case["rot"], "flops": 3 * case["n"] * case["heads"] * case["rot"]}
    stored = case["hd"] + case["hd"] // 16                     # bytes of a token of one kv head, keys and values
    if op == "append":
        values, slots = 2 * case["n"] * case["hkv"] * case["hd"], case["n"] * (case["hkv"] if case["per_head"] else 1)
        return {"bytes": 2 * values * _size(case) + case["n"] * case["hkv"] * stored + 4 * slots, "flops": 4 * values}
    heads, rows = _lengths(case)
    if op == "attention":
        tokens = sum(t + n for h, n in zip(heads, rows) for t in h)                        # over the kv heads
        pairs = sum(n * t + n * (n + 1) // 2 for h, n in zip(heads, rows) for t in h) * (case["hq"] // case["hkv"])
        per_row = case["hq"] * (2 * case["hd"] * _size(case) + 4)
        return {"bytes": tokens * (stored + (8 if case["weight"] else 0)) + sum(rows) * per_row, "flops": 4 * pairs * case["hd"]}
    held = moved = 0.0
    for h, budgets in zip(heads, _budgets(case)):
        for t, b in zip(h, budgets):
            new = min(t, b)
            newest = min(case["recent"], new, t - new)         # those of the newest that lie behind the new length: all of them stay
            free = max(0, new - case["recent"] - case["sinks"])
            held += t
            moved += newest + free * (t - new - newest) / max(1, t - case["recent"] - case["sinks"])
    return {"bytes": 8 * held + 2 * moved * (stored + 8) + 8 * case["reqs"] * case["hkv"], "flops": held}


# ---- the definitions in 64 bits ----

def _exact_power(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_values(codes, scales):
    lo, hi = codes & 15, codes >> 4
    code = torch.stack([lo, hi], dim=-1).flatten(-2)
    grid = torch.tensor(GRID, dtype=torch.float64, device=codes.device)
    x = grid[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0).double()
    return x * _exact_power(scales.long() - 127).repeat_interleave(32, dim=-1)


def _exact_rounded(x):
    """The nearest of the values that a group of 32 can hold: the step that the largest needs, ties to the even code."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(dim=-1, keepdim=True)
    e = torch.frexp(top.clamp(min=2.0**-140)).exponent - 3
    e = torch.where(top > 7.0 * _exact_power(e), e + 1, e).clamp(-124, 125)
    step = _exact_power(e)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    y = (x / step).abs()
    found = torch.zeros_like(y)
    best = (y - grid[0]).abs()
    for c in range(1, 8):
        d = (y - grid[c]).abs()
        nearer = (d < best) | ((d == best) & (c % 2 == 0))
        found, best = torch.where(nearer, grid[c], found), torch.where(nearer, d, best)
    return (found * step * torch.sign(x)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    op, hd = case["op"], case["hd"]
    if op == "rotary":
        n, heads, rot = case["n"], case["heads"], case["rot"]
        x = s.x[:, :heads * hd].double().reshape(n, heads, hd)
        turn = s.positions.double()[:, None, None] * _frequencies(case).to(DEV) * (-1.0 if case["inverse"] else 1.0)
        first = torch.arange(0, rot, 2) if case["interleaved"] else torch.arange(rot // 2)
        second = first + 1 if case["interleaved"] else first + rot // 2
        z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(turn, s.magnitude), turn)
        x[..., first], x[..., second] = z.real, z.imag
        return {"out": x.view(n, heads * hd)}
    if op == "append":
        shape = (case["n"], case["hkv"], hd)
        there = (s.slots >= 0) if case["per_head"] else (s.slots >= 0)[:, None]
        return {name: torch.where(there[..., None], _exact_rounded(x.view(shape)), 0.0).view(case["n"], -1) for name, x in (("k", s.k_new), ("v", s.v_new))}
    heads, rows = _lengths(case)
    if op == "attention":
        group = case["hq"] // case["hkv"]
        out = torch.empty(s.q.shape, dtype=torch.float64, device=DEV)
        lse = torch.empty(s.lse.shape, dtype=torch.float64, device=DEV)
        weight = s.weight.double() if case["weight"] else None
        at = 0
        for r, (lens, n) in enumerate(zip(heads, rows)):
            total = max(lens) + n
            block, off = _places(s, r, total)
            k, v = (_exact_values(c[block, :, off], e[block, :, off]).transpose(0, 1) for c, e in ((s.k, s.k_scale), (s.v, s.v_scale)))    # [hkv, total, hd]
            q = s.q[at:at + n].double().view(n, case["hkv"], group, hd).permute(1, 2, 0, 3)
            last = _int(lens).long()[:, None] + torch.arange(n, device=DEV)
            seen = torch.arange(total, device=DEV) <= last[:, :, None]
            x = torch.matmul(q, k.transpose(1, 2).contiguous()[:, None]) * s.scale
            x = torch.where(seen[:, None], x, -math.inf)
            norm = torch.logsumexp(x, dim=-1)
            p = torch.exp(x - norm[..., None])
            out[at:at + n] = torch.matmul(p, v[:, None]).permute(2, 0, 1, 3).reshape(n, -1)
            lse[at:at + n] = norm.permute(2, 0, 1).reshape(n, -1)
            if weight is not None:
                weight[block, :, off] += p.sum(dim=(1, 2)).T
            at += n
        found = {"out": out, "lse": lse}
        if weight is not None:
            found["weight"] = weight
        return found
    for r, (lens, budgets) in enumerate(zip(heads, _budgets(case))):
        block, off = _places(s, r, lens[0])
        for h, budget in enumerate(budgets):
            t, new = lens[0], min(lens[0], budget)
            w, p = s.weight[block, h, off].tolist(), s.position[block, h, off].tolist()
            rank = lambda i: (3, -p[i]) if p[i] < case["sinks"] else (2, p[i]) if p[i] >= 2 * t - case["recent"] else (1, w[i])
            kept = set(sorted(range(t), key=lambda i: (*rank(i), -i), reverse=True)[:new])
            s.new_lens[r, h] = new
            to, frm = [i for i in range(new) if i not in kept], [i for i in sorted(kept) if i >= new]
            for x in (s.k, s.v, s.k_scale, s.v_scale, s.weight, s.position):
                x[block[to], h, off[to]] = x[block[frm], h, off[frm]]
    s.weight = s.weight.double()
    return _evicted(s)
