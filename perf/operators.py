"""Timed cases of the operators at the two ends of a model: token ids in, token log-probabilities out, and back.

  embed       rows of the embedding table for a batch of token ids, scaled
  embed_grad  the table's gradient from the rows' gradients: one sum for every token of the batch
  logprobs    from rows of logits: the log-probability of one given token, the entropy, the best alternatives
  logprobs_grad  the gradient of those log-probabilities and entropies with respect to the logits

With `own` false each is computed in its plain form (elementary torch operations, fp32 inside), with `own` true by the
library's entry points.  A token id outside the vocabulary stands for padding: its row is zero and has no gradient.  A logit
of -inf bans its token."""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
LOWEST = float(torch.finfo(torch.float32).min)
RMS_EPS, ROPE_THETA = 1e-6, 1e4
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _embed(name, n, d, vocab, dtype, scale, pad=0.0):
    return dict(name=name, op="embed", n=n, d=d, vocab=vocab, dtype=dtype, scale=scale, pad=pad)


def _embed_grad(name, n, d, vocab, accumulate, scale=1.0, pad=0.0):
    return dict(name=name, op="embed_grad", n=n, d=d, vocab=vocab, accumulate=accumulate, scale=scale, pad=pad)


def _logprobs(name, n, vocab, dtype, ld=0, entropy=True, top_k=0, banned=0.0):
    return dict(name=name, op="logprobs", n=n, vocab=vocab, ld=ld or vocab, dtype=dtype, entropy=entropy, top_k=top_k, banned=banned)


def _logprobs_grad(name, n, vocab, dtype, out, ld=0, entropy=False, banned=0.0):
    return dict(name=name, op="logprobs_grad", n=n, vocab=vocab, ld=ld or vocab, dtype=dtype, out=out, entropy=entropy, banned=banned)


def listed():
    return [
        # the new tokens of a decode-only iteration of the edge configuration: one small launch
        _embed("embed_decode_edge", 32, 2048, 32000, "bf16", 1.0),
        # all rows of an iteration of the fp32 configuration, a few of them padding
        _embed("embed_tiny_fp32", 245, 256, 2048, "fp32", 16.0, pad=0.05),
        # all rows of the fine-tune-heavy iteration, scaled by the root of the width
        _embed("embed_7b_ft", 66576, 4096, 32000, "bf16", 64.0),
        # full fine-tuning of the edge configuration: the lookup's part of the tied table's gradient on top of the head's
        _embed_grad("embed_grad_edge_tied", 3347, 2048, 32000, True),
        # an untied table of the 7B-class model: the whole gradient is written
        _embed_grad("embed_grad_7b_table", 12288, 4096, 32000, False, pad=0.1),
        # the fine-tune-heavy iteration: frequent tokens fill thousands of rows
        _embed_grad("embed_grad_7b_ft_tied", 65536, 4096, 32000, True),
        # a server's answer to one request: the chosen token's log-probability and five alternatives
        _logprobs("logprobs_decode_one", 1, 32000, "fp32", top_k=5),
        # a decode batch, a quarter of its requests held to a grammar that bans most tokens
        _logprobs("logprobs_decode_7b", 256, 32000, "fp32", top_k=20, banned=0.9),
        # reference log-probabilities of all response tokens of the fine-tune-heavy iteration
        _logprobs("logprobs_reference_7b_ft", 32768, 32000, "fp32", entropy=False),
        # scoring with a large, odd vocabulary in a padded head, logits kept in bf16
        _logprobs("logprobs_score_bf16", 2048, 128011, "bf16", ld=128064, top_k=8),
        # gradient of the response tokens' log-probabilities as the operand of the head's weight gradient
        _logprobs_grad("logprobs_grad_7b_ft", 16384, 32000, "fp32", "bf16"),
        # an entropy bonus beside them on a small batch with an odd vocabulary, rows not aligned
        _logprobs_grad("logprobs_grad_entropy", 517, 31999, "fp32", "fp32", entropy=True, banned=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "logprobs", "logprobs", "logprobs_grad"))
    d = 64 * _log_int(rng, 2, 128)
    vocab = 64 * _log_int(rng, 8, 2000)
    if op == "embed":
        n = _log_int(rng, 1, min(66576, 66576 * 4096 // d))
        c = _embed("", n, d, vocab, rng.choice(("fp32", "bf16", "bf16")), rng.choice((1.0, math.sqrt(d))), rng.choice((0.0, 0.1)))
        if c["dtype"] == "fp32":
            c["n"] = max(1, n // 2)
    elif op == "embed_grad":
        accumulate = rng.random() < 0.5
        vocab = min(vocab, 64 * (32000 * 4096 // d // 64)) if not accumulate else vocab
        n = _log_int(rng, 1, min(65536, 65536 * 4096 // d // 2))
        c = _embed_grad("", n, d, vocab, accumulate, rng.choice((1.0, 1.0, math.sqrt(d))), rng.choice((0.0, 0.1)))
    else:
        vocab = _log_int(rng, 500, 128000)
        ld = vocab + rng.choice((0, 0, -vocab % 64, rng.randrange(1, 40)))
        dtype = rng.choice(("fp32", "fp32", "bf16"))
        banned = rng.choice((0.0, 0.0, 0.5, 0.9))
        if op == "logprobs":
            top_k = rng.choice((0, 1, 5, 20, 32))
            most = 3 * 10**8 if top_k else 5 * 10**8
            c = _logprobs("", _log_int(rng, 1, min(32768, most // vocab)), vocab, dtype, ld, rng.random() < 0.7, top_k, banned)
        else:
            c = _logprobs_grad("", _log_int(rng, 1, min(16384, 4 * 10**8 // vocab)), vocab, dtype, rng.choice(("fp32", "bf16", "bf16")), ld,
                               rng.random() < 0.5, banned)
    del c["name"]
    return c


def _frequencies(vocab):
    """Share of each token of a text: falls with the token's rank, the first few tokens make up a tenth of it."""
    w = 1.0 / (np.arange(vocab, dtype=np.float64) + 3.0)
    return w / w.sum()


def _ids(case, gen):
    """Token ids of text: frequent tokens scattered over the vocabulary, some rows padding (-1)."""
    cdf = torch.from_numpy(np.cumsum(_frequencies(case["vocab"]))).to(DEV)
    u = torch.rand(case["n"], generator=gen, device=DEV, dtype=torch.float64)
    rank = torch.searchsorted(cdf, u).clamp(max=case["vocab"] - 1)
    ids = torch.randperm(case["vocab"], generator=gen, device=DEV)[rank].int()
    if case["pad"]:
        ids[torch.rand(case["n"], generator=gen, device=DEV) < case["pad"]] = -1
    return ids


def _logits(case, gen):
    """Rows of logits of spread 1 to 4, in half of them one token far ahead as in a confident model; a quarter of the rows with
    banned tokens where the case has them, and the last of several such rows with every token banned."""
    n, vocab = case["n"], case["vocab"]
    x = torch.randn((n, case["ld"]), generator=gen, device=DEV)
    x *= 1.0 + 3.0 * torch.rand((n, 1), generator=gen, device=DEV)
    ahead = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    x[torch.arange(n, device=DEV), ahead] += 15.0 * (torch.rand(n, generator=gen, device=DEV) - 0.5).clamp(min=0.0) * 2.0
    # the given token: mostly the one that was ahead, else any; a few rows padding
    token = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.6, ahead, torch.randint(0, vocab, (n,), generator=gen, device=DEV)).int()
    if case["banned"]:
        rows = torch.arange(3, n, 4, device=DEV)
        for_rows = torch.rand((len(rows), case["ld"]), generator=gen, device=DEV) < case["banned"]
        x[rows] = x[rows].masked_fill(for_rows, -math.inf)
        if n > 8:
            x[n - 1] = -math.inf
    token[torch.rand(n, generator=gen, device=DEV) < 0.02] = -1
    return x.to(DTYPES[case["dtype"]]), token


class _Handle:
    def __init__(self, d, vocab, bf16):
        from paper_2510_03283_amd import binding as B
        self.B = B
        self.h = B.mace_create(d, d // 64, d // 64, 64, 64, vocab, RMS_EPS, ROPE_THETA, B.MACE_BF16 if bf16 else B.MACE_F32)

    def __del__(self):
        self.B.mace_destroy(self.h)


class _State:
    pass


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = _State()
    s.case, n, vocab = case, case["n"], case["vocab"]
    work_bytes = 0
    if own:
        # a handle is made once for a model; the head's operators go by the sizes of the call
        if case["op"].startswith("embed"):
            s.handle = _Handle(case["d"], vocab, case.get("dtype", "bf16") == "bf16")
        else:
            s.handle = _Handle(4096, 32000, True)
    if case["op"] == "embed":
        dtype = DTYPES[case["dtype"]]
        s.table = (0.02 * torch.randn((vocab, case["d"]), generator=gen, device=DEV)).to(dtype)
        s.ids = _ids(case, gen)
        s.out = torch.empty((n, case["d"]), dtype=dtype, device=DEV)
    elif case["op"] == "embed_grad":
        s.ids = _ids(case, gen)
        s.dx = 1e-3 * torch.randn((n, case["d"]), generator=gen, device=DEV)
        s.d_table = 1e-3 * torch.randn((vocab, case["d"]), generator=gen, device=DEV)
        if own:
            work_bytes = s.handle.B.mace_embed_grad_workspace_bytes(s.handle.h, n)
    else:
        s.x, s.token = _logits(case, gen)
        f32 = lambda *shape: torch.empty(shape, dtype=torch.float32, device=DEV)
        if case["op"] == "logprobs":
            k = case["top_k"]
            s.logp, s.stats = f32(n), f32(n, 2)
            s.entropy = f32(n) if case["entropy"] else None
            s.top_ids = torch.empty((n, k), dtype=torch.int32, device=DEV) if k else None
            s.top_logp = f32(n, k) if k else None
            if own:
                work_bytes = s.handle.B.mace_token_logprobs_workspace_bytes(s.handle.h, n, vocab, k)
        else:
            # what the forward left behind, and the gradients that come in: policy-gradient weights, an entropy bonus
            s.stats, s.entropy = _stats(s.x[:, :vocab].float(), case["entropy"])
            s.d_logp = torch.randn(n, generator=gen, device=DEV)
            s.d_entropy = -0.01 * torch.rand(n, generator=gen, device=DEV) if case["entropy"] else None
            s.d_x = torch.empty((n, vocab), dtype=DTYPES[case["out"]], device=DEV)
    s.work = torch.empty(max(work_bytes, 256), dtype=torch.uint8, device=DEV)
    return s


def _stats(x, entropy):
    """(max, log of the sum relative to it) of each row, and its entropy; a row without any finite logit: (-inf, 0), 0."""
    top = x.amax(dim=1, keepdim=True)
    t = x - top.clamp(min=LOWEST)
    e = t.exp()
    total = e.sum(dim=1, keepdim=True)
    empty = top[:, 0] == -math.inf
    log_sum = torch.where(empty, 0.0, total[:, 0].log())
    h = None
    if entropy:
        h = log_sum - (e * t.clamp(min=LOWEST)).sum(dim=1) / torch.where(empty, 1.0, total[:, 0])
    return torch.stack([top[:, 0], log_sum], dim=1), h


def _best(x, k):
    """Columns of the k largest values of each row, ties to the lower column; -1 where only banned tokens are left."""
    bits = (x + 0.0).view(torch.int32)                      # -0 counts as 0
    ordered = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    column = torch.arange(x.shape[1], device=x.device)
    key = (ordered << 32) | (0xFFFFFFFF - column)
    best = key.topk(min(k, x.shape[1]), dim=1).values
    ids = 0xFFFFFFFF - (best & 0xFFFFFFFF)
    values = x.gather(1, ids)
    gone = values == -math.inf
    return ids.masked_fill(gone, -1).int(), values


def _plain_logprobs(s):
    case = s.case
    x = s.x[:, :case["vocab"]].float()
    stats, entropy = _stats(x, case["entropy"])
    top, log_sum = stats[:, 0].clamp(min=LOWEST), stats[:, 1]
    given = (s.token >= 0) & (s.token < case["vocab"])
    own_x = x.gather(1, torch.where(given, s.token, 0).long()[:, None])[:, 0]
    logp = torch.where(given, own_x - top - log_sum, 0.0)
    out = {"logp": logp, "stats": stats}
    if case["entropy"]:
        out["entropy"] = entropy
    if case["top_k"]:
        ids, values = _best(x, case["top_k"])
        out["top_ids"], out["top_logp"] = ids, values - top[:, None] - log_sum[:, None]
    return out


def _plain_logprobs_grad(s):
    case = s.case
    x = s.x[:, :case["vocab"]].float()
    top, log_sum = s.stats[:, :1].clamp(min=LOWEST), s.stats[:, 1:]
    lp = x - top - log_sum
    p = lp.exp()
    given = (s.token >= 0) & (s.token < case["vocab"])
    g = torch.where(given, s.d_logp, 0.0)
    grad = -g[:, None] * p
    grad.scatter_add_(1, torch.where(given, s.token, 0).long()[:, None], g[:, None])
    if case["entropy"]:
        grad -= s.d_entropy[:, None] * p * (lp.clamp(min=LOWEST) + s.entropy[:, None])
    grad = torch.where(s.stats[:, :1] == -math.inf, 0.0, grad)
    return {"d_logits": grad.to(DTYPES[case["out"]])}


def _plain_embed(s):
    there = s.ids >= 0
    rows = s.table[torch.where(there, s.ids, 0).long()].float() * s.case["scale"]
    return {"out": torch.where(there[:, None], rows, 0.0).to(s.table.dtype)}


def _plain_embed_grad(s):
    there = s.ids >= 0
    dx = torch.where(there[:, None], s.dx, 0.0) * s.case["scale"]
    ids = torch.where(there, s.ids, 0).long()
    if not s.case["accumulate"]:
        s.d_table.zero_()
    s.d_table.index_add_(0, ids, dx)
    return {"d_table": s.d_table}


def run(s):
    op, case = s.case["op"], s.case
    if not own:
        return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "logprobs": _plain_logprobs, "logprobs_grad": _plain_logprobs_grad}[op](s)
    B, h = s.handle.B, s.handle.h
    if op == "embed":
        B.mace_embed_tokens(h, s.table, s.ids, s.out, case["scale"])
        return {"out": s.out}
    if op == "embed_grad":
        B.mace_embed_tokens_grad(h, s.ids, s.dx, s.d_table, s.work, case["scale"], case["accumulate"])
        return {"d_table": s.d_table}
    if op == "logprobs":
        B.mace_token_logprobs(h, s.x, s.work, s.token, s.logp, s.entropy, s.stats, s.top_ids, s.top_logp, case["vocab"])
        out = {"logp": s.logp, "stats": s.stats}
        if case["entropy"]:
            out["entropy"] = s.entropy
        if case["top_k"]:
            out["top_ids"], out["top_logp"] = s.top_ids, s.top_logp
        return out
    B.mace_token_logprobs_grad(h, s.x, s.stats, s.d_x, s.token, s.d_logp, s.entropy, s.d_entropy, case["vocab"])
    return {"d_logits": s.d_x}


def _size(dtype):
    return 4 if dtype == "fp32" else 2


def work(case):
    n, vocab = case["n"], case["vocab"]
    if case["op"].startswith("embed"):
        d = case["d"]
        there = n * (1.0 - case["pad"])
        distinct = float(np.sum(-np.expm1(there * np.log1p(-_frequencies(vocab)))))     # tokens that occur at all
        if case["op"] == "embed":
            return {"bytes": 4 * n + (distinct + n) * d * _size(case["dtype"]), "flops": n * d}
        table = 2 * distinct if case["accumulate"] else vocab
        return {"bytes": 4 * n + 4 * d * (there + table), "flops": 2 * there * d}
    cells = n * vocab
    if case["op"] == "logprobs":
        per_row = 4 + 4 + 8 + (4 if case["entropy"] else 0) + 8 * case["top_k"]
        return {"bytes": cells * _size(case["dtype"]) + n * per_row, "flops": cells * (6 if case["entropy"] else 4)}
    return {"bytes": cells * (_size(case["dtype"]) + _size(case["out"])) + 24 * n, "flops": cells * (8 if case["entropy"] else 4)}


def _exact_rows(x, token, entropy, k):
    """logp, stats, entropy, ids, top_logp of rows of fp64 logits, by sorting."""
    empty = torch.isneginf(x).all(dim=1)
    lse = torch.logsumexp(x, dim=1)
    top = x.max(dim=1).values
    out = {"stats": torch.stack([top, torch.where(empty, 0.0, lse - top)], dim=1)}
    lp = torch.where(empty[:, None], -math.inf, x - lse[:, None])
    given = (token >= 0) & (token < x.shape[1])
    out["logp"] = torch.where(given, lp.gather(1, token.clamp(0, x.shape[1] - 1).long()[:, None])[:, 0], 0.0)
    if entropy:
        out["entropy"] = torch.special.entr(lp.exp()).sum(dim=1)
    if k:
        values, ids = lp.sort(dim=1, descending=True, stable=True)
        width = min(k, x.shape[1])
        out["top_ids"] = torch.where(torch.isneginf(values[:, :width]), -1, ids[:, :width]).int()
        out["top_logp"] = values[:, :width]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    n, vocab = case["n"], case["vocab"]
    if case["op"] == "embed":
        padded = torch.cat([s.table.double(), torch.zeros((1, case["d"]), dtype=torch.float64, device=DEV)])
        return {"out": padded[torch.where(s.ids < 0, vocab, s.ids).long()] * case["scale"]}
    if case["op"] == "embed_grad":
        total = torch.zeros((vocab + 1, case["d"]), dtype=torch.float64, device=DEV)
        total.index_add_(0, torch.where(s.ids < 0, vocab, s.ids).long(), s.dx.double())
        total = total[:vocab] * case["scale"]
        return {"d_table": total + s.d_table.double() if case["accumulate"] else total}
    rows = max(1, 2**27 // vocab)
    parts = []
    for r in range(0, n, rows):
        x, token = s.x[r:r + rows, :vocab].double(), s.token[r:r + rows]
        if case["op"] == "logprobs":
            parts.append(_exact_rows(x, token, case["entropy"], case["top_k"]))
            continue
        live = ~torch.isneginf(x).all(dim=1, keepdim=True)
        p = torch.where(live, torch.softmax(torch.where(live, x, 0.0), dim=1), 0.0)
        given = ((token >= 0) & (token < vocab))[:, None] & live
        pick = torch.zeros_like(p).scatter_(1, token.clamp(0, vocab - 1).long()[:, None], given.double())
        grad = s.d_logp[r:r + rows, None].double() * torch.where(given, pick - p, 0.0)
        if case["entropy"]:
            surprise = torch.where(p > 0, -p.log(), 0.0)
            mean = (p * surprise).sum(dim=1, keepdim=True)
            grad += s.d_entropy[r:r + rows, None].double() * p * (surprise - mean)
        parts.append({"d_logits": grad})
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
