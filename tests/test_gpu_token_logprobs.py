"""Token log-probabilities, entropies, alternatives and their gradients through the C ABI against their definitions in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24                        # half a step of fp32, relative
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
INF = math.inf
LOWEST = -3.4028234663852886e38


@pytest.fixture(scope="module")
def lib(torch_mod):
    from paper_2510_03283_amd import binding as B
    h = B.mace_create(256, 4, 4, 64, 704, 2048, 1e-6, 1e4, B.MACE_BF16)
    yield B, h
    B.mace_destroy(h)


def workspace(torch, lib, n, vocab, k):
    """Scratch that holds NaNs and wild indices: nothing in it may be read before it is written."""
    return torch.full((lib[0].mace_token_logprobs_workspace_bytes(lib[1], n, vocab, k),), 0xFF, dtype=torch.uint8, device="cuda")


def rows_of(torch, x, ld, offset, dtype):
    """x as rows that lie ld elements apart, the first one `offset` elements into an allocation that holds NaN everywhere else."""
    n, vocab = x.shape
    buf = torch.full((offset + max(n - 1, 0) * ld + vocab + 64,), float("nan"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    view = buf[offset:].as_strided((n, vocab), (ld, 1))
    view.copy_(x)
    return view


def call(torch, lib, x, token=None, k=0, ws=None, vocab=None, stream=None):
    B, h = lib
    n, V = x.shape[0], vocab or x.shape[1]
    f = lambda *s: torch.full(s, 123.0, dtype=torch.float32, device="cuda")
    o = dict(logp=f(n) if token is not None else None, entropy=f(n), row_stats=f(n, 2),
             top_ids=torch.full((n, k), -99, dtype=torch.int32, device="cuda") if k else None, top_logp=f(n, k) if k else None)
    B.mace_token_logprobs(h, x, workspace(torch, lib, n, V, k) if ws is None else ws, token, vocab=vocab, stream=stream, **o)
    return o


def check(torch, x, token, o, k):
    """x: the logits as stored (rows without NaN or +inf)."""
    n, vocab = x.shape
    for r0 in range(0, n, max(1, 2**25 // vocab)):
        r = slice(r0, min(n, r0 + max(1, 2**25 // vocab)))
        x64 = x[r].double()
        m = x64.max(dim=1, keepdim=True).values
        empty = torch.isneginf(m[:, 0])
        t = torch.where(torch.isneginf(x64), -INF, x64 - torch.where(empty[:, None], 0.0, m))
        e = t.exp()
        s = e.sum(dim=1)
        ok = ~empty
        L = torch.where(ok, s.log(), 0.0)
        lp = torch.where(ok[:, None], t - L[:, None], -INF)
        tt = torch.where(e > 0, t.abs(), 0.0)
        # Error of the sums: e^t has 3 |t| half steps from t and its product with log2 e, 4 of the exponential; a sum of vocab terms by
        # 256 threads or more and a tree has a depth of at most vocab / 256 + 32 additions (and as many rescalings by a further factor).
        depth = 2 * (vocab / 256 + 32)
        s_ = torch.where(ok, s, 1.0)
        tbar, t2bar = (e * tt).sum(dim=1) / s_, (e * tt * tt).sum(dim=1) / s_
        rel_s = EPS * (3 * tbar + depth + 4)
        stats = o["row_stats"][r].double()
        assert torch.equal(stats[:, 0], m[:, 0])
        # an error of the sum moves L by as much; where L is near 0 its own logarithm has a rounding of 1 + (L)
        tol_L = rel_s + EPS * (4 + 2 * L.abs())
        assert ((stats[:, 1] - L).abs() <= tol_L).all()
        if o["logp"] is not None:
            given = (token[r] >= 0) & (token[r] < vocab)
            at = token[r].clamp(0, vocab - 1).long()[:, None]
            want = torch.where(given, lp.gather(1, at)[:, 0], 0.0)
            got = o["logp"][r].double()
            fin = torch.isfinite(want)
            assert torch.equal(got[~fin], want[~fin])
            slack = tol_L + EPS * 2 * (tt.gather(1, at)[:, 0] + L.abs() + 1)
            assert ((got - want).abs() <= slack)[fin].all()
        H = torch.where(ok, L + (e * tt).sum(dim=1) / s_, 0.0)
        tol_H = tol_L + EPS * (3 * t2bar + (depth + 8) * tbar) + tbar * rel_s + EPS * 4 * H
        assert ((o["entropy"][r].double() - H).abs() <= torch.where(ok, tol_H, 0.0)).all()
        if k:
            order = x[r].float().sort(dim=1, descending=True, stable=True)
            w = min(k, vocab)
            ids, val = order.indices[:, :w], order.values[:, :w].double()
            gone = torch.isneginf(val)
            want_ids = torch.full((ids.shape[0], k), -1, device="cuda")
            want_ids[:, :w] = torch.where(gone, -1, ids)
            assert torch.equal(o["top_ids"][r].long(), want_ids)
            want = torch.full((ids.shape[0], k), -INF, dtype=torch.float64, device="cuda")
            want[:, :w] = lp.gather(1, ids)
            got, fin = o["top_logp"][r].double(), torch.isfinite(want)
            assert torch.equal(got[~fin], want[~fin])
            slack = tol_L[:, None] + EPS * 2 * ((want + L[:, None]).abs() + L[:, None].abs() + 1)
            assert ((got - want).abs() <= slack)[fin].all()


def draw(torch, n, vocab, kind, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, vocab), generator=gen, device="cuda") * (0.5 + 4 * torch.rand((n, 1), generator=gen, device="cuda"))
    if kind == "peaked":
        x[torch.arange(n, device="cuda"), torch.randint(0, vocab, (n,), generator=gen, device="cuda")] += 5.0 + 30.0 * torch.rand(n, generator=gen, device="cuda")
    elif kind == "banned":              # from no banned token to all but a few, and one row with nothing left
        x = x.masked_fill(torch.rand((n, vocab), generator=gen, device="cuda") < torch.linspace(0, 1.001, n, device="cuda")[:, None] ** 0.25, -INF)
        x[n // 2] = -INF
    elif kind == "lowest":              # bans by the lowest value: ordinary logits that many columns share
        x = x.masked_fill(torch.rand((n, vocab), generator=gen, device="cuda") < 0.999, LOWEST)
        x[n // 2] = LOWEST
    elif kind == "equal":
        x = torch.arange(n, device="cuda")[:, None].float().expand(n, vocab).clone() - 3
    elif kind == "coarse":              # few distinct values: ties everywhere, also of -0 and +0
        x = (x / 2).round() * torch.where(torch.rand((n, vocab), generator=gen, device="cuda") < 0.5, 1.0, -1.0)
    elif kind == "rising":
        x = torch.linspace(-20, 20, vocab, device="cuda").expand(n, vocab).clone()
    elif kind == "falling":
        x = torch.linspace(20, -20, vocab, device="cuda").expand(n, vocab).clone()
    elif kind == "large":               # differences of a few at magnitudes of ten thousands
        x = x + 30000.0 * torch.randint(-1, 2, (n, 1), generator=gen, device="cuda")
    token = torch.randint(0, vocab, (n,), generator=gen, device="cuda").int()
    token[::5] = x[::5].argmax(dim=1).int()
    token[3::7] = torch.tensor([-1, vocab, -2**31, 2**31 - 1], device="cuda").repeat(n)[:len(token[3::7])].int()
    return x, token


SHAPES = [(1, 1), (2, 3), (5, 64), (9, 255), (3, 1000), (17, 2048), (300, 777), (1, 32000), (40, 32000), (600, 4099), (2, 128011), (33, 50001), (1000, 33001), (1400, 50001)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,vocab", SHAPES)
def test_sizes(torch_mod, lib, dtype, n, vocab):
    torch = torch_mod
    x, token = draw(torch, n, vocab, "peaked" if n % 2 else "plain", n + vocab)
    # aligned rows; rows of odd stride; rows that start an element off an aligned address
    for ld, offset, k in ((vocab + -vocab % 64, 0, 5), (vocab + (vocab % 2 == 0), 0, 32), (vocab, 1, 0), (vocab + 7, 3, 20)):
        rows = rows_of(torch, x, ld, offset, dtype)
        o = call(torch, lib, rows, token, k)
        torch.cuda.synchronize()
        check(torch, rows, token, o, k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "peaked", "banned", "lowest", "equal", "coarse", "rising", "falling", "large"])
@pytest.mark.parametrize("n,vocab,k", [(12, 70, 32), (37, 2048, 20), (21, 31999, 32), (7, 131072, 8), (1100, 1003, 4), (300, 12301, 20), (9, 6145, 24), (1000, 33001, 20)])
def test_values(torch_mod, lib, dtype, kind, n, vocab, k):
    torch = torch_mod
    x, token = draw(torch, n, vocab, kind, 11 + n)
    rows = rows_of(torch, x, vocab, 0, dtype)
    o = call(torch, lib, rows, token, k)
    torch.cuda.synchronize()
    check(torch, rows, token, o, k)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(8, 130), (8, 5000), (2100, 700), (8, 131072)])
def test_magnitudes(torch_mod, lib, dtype, n, vocab):
    """Logits around every magnitude, one to a row, up to the largest; differences of a few there where the type has them."""
    torch = torch_mod
    x, token = draw(torch, n, vocab, "plain", 5)
    centre = torch.tensor([0.0, 9.0e5, -9.0e5, 2.0e6, -2.0e6, 1e30, -1e30, 3e38], device="cuda").repeat(n // 8 + 1)[:n, None]
    x = x + centre
    x[1::8, ::3] = LOWEST                                                    # far below the rest, but allowed
    x[2::8, ::3] = -INF
    rows = rows_of(torch, x, vocab, 0, dtype)
    o = call(torch, lib, rows, token, 6)
    torch.cuda.synchronize()
    check(torch, rows, token, o, 6)


@pytest.mark.parametrize("rest", [-INF, LOWEST])
def test_one_allowed_token_in_a_long_row(torch_mod, lib, rest):
    """Rows that several blocks share, with everything in one of them."""
    torch = torch_mod
    n, vocab = 5, 128011
    x = torch.full((n, vocab), rest, device="cuda")
    at = torch.tensor([0, 40000, 65535, 100000, vocab - 1], device="cuda")
    x[torch.arange(n), at] = torch.tensor([1.0, -3.0, 0.0, 30.0, -200.0], device="cuda")
    token = at.int()
    token[2] = 7
    o = call(torch, lib, x, token, 4)
    torch.cuda.synchronize()
    check(torch, x, token, o, 4)
    assert torch.equal(o["top_ids"][:, 0].long(), at) and (o["entropy"] == 0).all()


def test_very_long_rows(torch_mod, lib):
    torch = torch_mod
    for n, vocab, dtype in ((3, 1 << 22, "fp32"), (600, 300001, "bf16")):
        x, token = draw(torch, n, vocab, "peaked", n)
        rows = rows_of(torch, x, vocab, 0, dtype)
        o = call(torch, lib, rows, token, 20)
        torch.cuda.synchronize()
        check(torch, rows, token, o, 20)


def test_offsets_past_32_bits(torch_mod, lib):
    """Rows that end 8.6 GB into their buffer: element offsets past 2^31."""
    torch = torch_mod
    vocab, ld, n = 1000, 33_000_001, 66
    buf = torch.empty(ld * (n - 1) + vocab, dtype=torch.float32, device="cuda")
    rows = buf.as_strided((n, vocab), (ld, 1))
    x, token = draw(torch, n, vocab, "peaked", 4)
    rows.copy_(x)
    o = call(torch, lib, rows, token, 5)
    torch.cuda.synchronize()
    check(torch, x, token, o, 5)
    want = torch.empty((n, vocab), device="cuda")
    ones = torch.ones(n, device="cuda")
    lib[0].mace_token_logprobs_grad(lib[1], rows, o["row_stats"], want, token, ones)
    lib[0].mace_token_logprobs_grad(lib[1], rows, o["row_stats"], rows, token, ones)          # in place
    torch.cuda.synchronize()
    assert torch.equal(rows, want)


def test_only_the_vocabulary_counts(torch_mod, lib):
    """Columns behind vocab (the padding of a head) hold NaN and +inf."""
    torch = torch_mod
    x, token = draw(torch, 40, 1001, "plain", 2)
    wide = torch.full((40, 1024), float("nan"), device="cuda")
    wide[:, 1010:] = INF
    wide[:, :1001] = x
    o = call(torch, lib, wide, token, 6, vocab=1001)
    d = torch.full((40, 1024), 5.0, device="cuda")
    lib[0].mace_token_logprobs_grad(lib[1], wide, o["row_stats"], d, token, torch.ones(40, device="cuda"), vocab=1001)
    torch.cuda.synchronize()
    check(torch, x, token, o, 6)
    assert torch.isfinite(d[:, :1001]).all() and (d[:, 1001:] == 5).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 2048, 40001, 128011])
def test_nan_and_infinity(torch_mod, lib, dtype, vocab):
    """A NaN or +inf makes its own row NaN and no other."""
    torch = torch_mod
    n = 30
    x, token = draw(torch, n, vocab, "plain", 8)
    token[:] = torch.arange(n, device="cuda") % vocab
    token[9::10] = -1
    x[::3, vocab // 2] = float("nan")
    x[1::6, vocab - 1] = INF
    x[4::12, 0] = -INF                                                       # an ordinary ban among them
    bad = torch.isnan(x).any(dim=1) | (x == INF).any(dim=1)
    x[2, :] = float("nan"); bad[2] = True
    rows = rows_of(torch, x, vocab, 0, dtype)
    o = call(torch, lib, rows, token, 3)
    d = torch.empty((n, vocab), device="cuda")
    weight = torch.ones(n, device="cuda")
    lib[0].mace_token_logprobs_grad(lib[1], rows, o["row_stats"], d, token, weight)
    torch.cuda.synchronize()
    good = ~bad
    sub = {k: v[good] for k, v in o.items()}
    check(torch, rows[good], token[good], sub, 3)
    given = token >= 0
    assert torch.isnan(o["logp"][bad & given]).all() and (o["logp"][~given] == 0).all()
    assert torch.isnan(o["entropy"][bad]).all() and torch.isnan(o["row_stats"][bad]).all()
    assert (o["top_ids"][bad] == -1).all() and torch.isnan(o["top_logp"][bad]).all()
    assert torch.isfinite(d[good]).all() and torch.isnan(d[bad & given]).all()
    assert (d[~given] == 0).all()                                            # padding: no weight, no gradient, whatever the logits hold


def test_outputs_one_by_one(torch_mod, lib):
    """Every output on its own has the bits that it has beside the others."""
    torch = torch_mod
    B, h = lib
    for n, vocab in ((3, 32000), (700, 2049)):
        x, token = draw(torch, n, vocab, "peaked", 1)
        o = call(torch, lib, x, token, 7)
        ws = workspace(torch, lib, n, vocab, 7)
        for names in (("logp",), ("entropy",), ("row_stats",), ("top_ids",), ("top_ids", "top_logp"), ("logp", "row_stats")):
            part = {k: torch.full_like(o[k], 77) for k in names}
            B.mace_token_logprobs(h, x, ws, token if "logp" in names else None, **part)
            torch.cuda.synchronize()
            for k in names:
                assert torch.equal(part[k], o[k]), (n, k)


def grad_check(torch, lib, x, token, dtype, out, entropy, logp, ld_out=None, in_place=False):
    B, h = lib
    n, vocab = x.shape
    o = call(torch, lib, x, token)
    gen = torch.Generator(device="cuda").manual_seed(n)
    g = torch.randn(n, generator=gen, device="cuda") if logp else None
    w = torch.randn(n, generator=gen, device="cuda") if entropy else None
    odt = torch.bfloat16 if out == "bf16" else torch.float32
    keep = x.clone()
    ld_out = ld_out or vocab
    buf = torch.full((n * ld_out + 16,), 9.0, dtype=odt, device="cuda")
    d = x if in_place else buf[:n * ld_out].view(n, ld_out)
    B.mace_token_logprobs_grad(h, x, o["row_stats"], d, token if logp else None, g, o["entropy"] if entropy else None, w, vocab=vocab)
    torch.cuda.synchronize()
    if not in_place:
        assert (d[:, vocab:] == 9).all() and (buf[n * ld_out:] == 9).all()
        assert torch.equal(x.view(torch.int16 if dtype == "bf16" else torch.int32), keep.view(torch.int16 if dtype == "bf16" else torch.int32))
    # the formula in 64 bits, on the statistics and entropies that the call was given
    x64, m, L = keep.double(), o["row_stats"][:, :1].double(), o["row_stats"][:, 1:].double()
    empty = torch.isneginf(m)
    t = torch.where(empty, -INF, x64 - torch.where(empty, 0.0, m))
    lp = t - L
    p = lp.exp()
    lp_, H = torch.where(p > 0, lp, 0.0), o["entropy"].double()[:, None]
    given = (token >= 0) & (token < vocab)
    g64 = torch.where(given, g.double(), 0.0)[:, None] if logp else torch.zeros((n, 1), dtype=torch.float64, device="cuda")
    w64 = w.double()[:, None] if entropy else torch.zeros_like(g64)
    one = torch.zeros_like(p).scatter_(1, token.clamp(0, vocab - 1).long()[:, None], given[:, None].double())
    want = torch.where(empty, 0.0, g64 * (one - p) - w64 * p * (lp_ + H))
    # lp: two subtractions, half a step each of t and lp; p: that and 3 half steps of lp log2 e, 4 of the exponential
    err_lp = EPS * (torch.where(p > 0, t.abs(), 0.0) + 2 * lp_.abs())
    err_p = p * (err_lp + EPS * (3 * lp_.abs() + 4))
    err = g64.abs() * err_p + w64.abs() * (err_p * (lp_ + H).abs() + p * (err_lp + EPS * (lp_.abs() + H)))
    err = err + EPS * 4 * (g64.abs() * (one + p) + w64.abs() * p * (lp_ + H).abs())
    # results below the smallest normal number may be flushed to zero
    bound = err + HALF[out] * (want.abs() + err) + 2 * 1.2e-38
    assert ((d[:, :vocab].double() - want).abs() <= bound).all()
    banned = torch.isneginf(keep) & (one == 0)                               # (a given token that is banned keeps its g)
    assert (d[:, :vocab][banned] == 0).all()


@pytest.mark.parametrize("dtype,out", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("n,vocab,ld,offset,ld_out", [(1, 1, 1, 0, 1), (7, 3, 5, 1, 4), (33, 255, 256, 0, 256), (12, 2048, 2048, 0, 2048), (21, 4097, 4099, 3, 4097),
                                                       (5, 32000, 32000, 0, 32064), (3, 128011, 128064, 0, 128011), (1500, 100, 100, 2, 100), (30, 9001, 9003, 1, 9005)])
def test_gradient(torch_mod, lib, dtype, out, n, vocab, ld, offset, ld_out):
    torch = torch_mod
    x, token = draw(torch, n, vocab, "banned" if n > 20 else "peaked", n)
    rows = rows_of(torch, x, ld, offset, dtype)
    for entropy, logp in ((True, True), (False, True), (True, False)):
        grad_check(torch, lib, rows, token, dtype, out, entropy, logp, ld_out)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_in_place(torch_mod, lib, dtype):
    torch = torch_mod
    for vocab, ld, offset in ((2048, 2048, 0), (1001, 1003, 1), (9001, 9003, 5)):
        x, token = draw(torch, 50, vocab, "banned", 6)
        rows = rows_of(torch, x, ld, offset, dtype)
        grad_check(torch, lib, rows, token, dtype, dtype, True, True, in_place=True)


@pytest.mark.parametrize("kind", ["lowest", "equal", "large", "coarse"])
def test_gradient_values(torch_mod, lib, kind):
    torch = torch_mod
    x, token = draw(torch, 20, 3001, kind, 6)
    grad_check(torch, lib, x, token, "fp32", "fp32", True, True)


def test_gradient_is_the_slope(torch_mod, lib):
    """Central differences of the forward, one column at a time.  With steps of 2^-6 the third derivatives (at most 1 for logp, 3 for the
    entropy of these rows) leave 2^-12 / 6 x 3 = 1.2e-4, the roundings of two results of at most 4 a step 4 x 2^-23 / 2^-6 = 3e-5."""
    torch = torch_mod
    n, vocab, step = 6, 9, 2.0 ** -6
    x, token = draw(torch, n, vocab, "plain", 12)
    x.clamp_(-2, 2)
    token = token.clamp(0, vocab - 1)
    o = call(torch, lib, x, token)
    for weights in (("d_logp",), ("d_entropy",)):
        d = torch.empty_like(x)
        w = {k: torch.ones(n, device="cuda") for k in weights}
        lib[0].mace_token_logprobs_grad(lib[1], x, o["row_stats"], d, token, entropy=o["entropy"], **w)
        for j in range(vocab):
            up, down = x.clone(), x.clone()
            up[:, j] += step
            down[:, j] -= step
            name = weights[0][2:]
            slope = (call(torch, lib, up, token)[name].double() - call(torch, lib, down, token)[name].double()) / (up[:, j] - down[:, j]).double()
            torch.cuda.synchronize()
            assert (slope - d[:, j].double()).abs().max() <= 1.5e-4, (weights, j)


def test_graph_and_streams(torch_mod, lib):
    """Captured on a side stream and replayed on new logits, eager calls in between: every replay gives the eager bits."""
    torch = torch_mod
    B, h = lib
    for n, vocab in ((2, 32000), (900, 1001)):
        x, token = draw(torch, n, vocab, "plain", 1)
        k = 9
        ws = workspace(torch, lib, n, vocab, k)
        o = call(torch, lib, x, token, k)
        d, g = torch.empty_like(x), torch.ones(n, device="cuda")
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            B.mace_token_logprobs(h, x, ws, token, **o)
            B.mace_token_logprobs_grad(h, x, o["row_stats"], d, token, g, o["entropy"], g)
        for turn in range(3):
            new, t = draw(torch, n, vocab, ("banned", "coarse", "peaked")[turn], turn)
            x.copy_(new)
            token.copy_(t)
            want = call(torch, lib, x, token, k, stream=torch.cuda.current_stream())
            want_d = torch.empty_like(x)
            B.mace_token_logprobs_grad(h, x, want["row_stats"], want_d, token, g, want["entropy"], g)
            torch.cuda.synchronize()
            for v in (*o.values(), d):
                v.fill_(55)
            ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o[key], want[key]) for key in o) and torch.equal(d, want_d), turn


def test_binding_refuses_what_the_library_cannot_see(torch_mod, lib):
    torch = torch_mod
    B, h = lib
    x, token = torch.zeros((4, 100), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ws, lp, st = workspace(torch, lib, 4, 100, 5), torch.zeros(4, device="cuda"), torch.zeros((4, 2), device="cuda")
    ids, tl = torch.zeros((4, 5), dtype=torch.int32, device="cuda"), torch.zeros((4, 5), device="cuda")
    good = dict(token_ids=token, logp=lp, row_stats=st, top_ids=ids, top_logp=tl)
    B.mace_token_logprobs(h, x, ws, **good)
    for bad in (dict(token_ids=token[:3]), dict(token_ids=token.long()), dict(logp=lp[:3]), dict(logp=lp.double()), dict(row_stats=st.view(-1)), dict(top_ids=ids[:3]),
                dict(top_ids=ids.long()), dict(top_logp=tl[:, :4].contiguous()), dict(top_ids=None), dict(vocab=101), dict(token_ids=token.cpu()),
                dict(top_ids=torch.zeros((4, 33), dtype=torch.int32, device="cuda"), top_logp=torch.zeros((4, 33), device="cuda"))):
        with pytest.raises(B.MaceError):
            B.mace_token_logprobs(h, x, ws, **{**good, **bad})
    for bad_x in (x.t(), x.half(), x[0], x.cpu(), x[:1].expand(4, 100)):
        with pytest.raises(B.MaceError):
            B.mace_token_logprobs(h, bad_x, ws, logp=lp, token_ids=token)
    with pytest.raises(B.MaceError):
        B.mace_token_logprobs(h, x, ws[:0], logp=lp, token_ids=token)
    d = torch.zeros((4, 100), device="cuda")
    for args in ((x, st[:3], d), (x, st, d[:3]), (x, st, d[:, :99]), (x, st, d.double()), (x, st, x[:, ::2])):
        with pytest.raises(B.MaceError):
            B.mace_token_logprobs_grad(h, *args, token, lp)
    with pytest.raises(B.MaceError):
        B.mace_token_logprobs_grad(h, x, st, d, token)
