"""Embedding rows and the table's gradient through the C ABI against their definitions."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
EPS32 = 2.0 ** -24                      # half a step of fp32, relative


class Model:
    """A handle of this table size (the other dimensions do not matter here)."""

    def __init__(self, d, vocab, bf16):
        from paper_2510_03283_amd import binding as B
        self.B, self.h = B, B.mace_create(d, 1, 1, 64, 64, vocab, 1e-6, 1e4, B.MACE_BF16 if bf16 else B.MACE_F32)

    def __enter__(self):
        return self.B, self.h

    def __exit__(self, *_):
        self.B.mace_destroy(self.h)


def workspace(torch, B, h, n):
    """Scratch that holds NaNs and wild indices: nothing in it may be read before it is written."""
    return torch.full((B.mace_embed_grad_workspace_bytes(h, n),), 0xFF, dtype=torch.uint8, device="cuda")


def draw_ids(torch, kind, n, vocab, seed):
    r = np.random.default_rng(seed)
    if kind == "uniform":
        ids = r.integers(0, vocab, n)
    elif kind == "text":                # frequent tokens, padding and ids from outside
        w = 1.0 / (np.arange(vocab) + 3.0)
        ids = r.permutation(vocab)[r.choice(vocab, n, p=w / w.sum())]
        ids[r.random(n) < 0.1] = -1
        ids[r.random(n) < 0.02] = vocab
        ids[r.random(n) < 0.02] = r.choice([-2**31, 2**31 - 1, vocab + 1])
    elif kind == "one":                 # every row the same token
        ids = np.full(n, vocab // 2)
    elif kind == "two":                 # the first and the last token of the table in turn
        ids = np.where(np.arange(n) % 2 == 0, 0, vocab - 1)
    elif kind == "padding":
        ids = np.full(n, -1)
    elif kind == "sorted":
        ids = np.sort(r.integers(0, vocab, n))
    elif kind == "runs":                # every token exactly 64 times, in turn
        ids = np.arange(n) % max(1, n // 64) % vocab
    return torch.from_numpy(ids.astype(np.int32)).cuda()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,d,vocab,scale", [(1, 64, 64, 1.0), (3, 128, 320, 8.0), (77, 256, 2048, 0.3), (1000, 2048, 32000, 1.0), (513, 4096, 1024, 64.0),
                                             (129, 8192, 640, -2.5), (5000, 192, 128000, 1.0), (260, 960, 704, 0.0)])
def test_rows(torch_mod, bf16, n, d, vocab, scale):
    torch = torch_mod
    gen = torch.Generator(device="cuda").manual_seed(n + d)
    table = torch.randn((vocab, d), generator=gen, device="cuda").to(torch.bfloat16 if bf16 else torch.float32)
    ids = draw_ids(torch, "text", n, vocab, n)
    out = torch.full((n + 2, d), 7.0, dtype=table.dtype, device="cuda")
    with Model(d, vocab, bf16) as (B, h):
        B.mace_embed_tokens(h, table, ids, out[1:n + 1], scale)
        torch.cuda.synchronize()
    there = (ids >= 0) & (ids < vocab)
    want = torch.zeros((n, d), dtype=table.dtype, device="cuda")
    want[there] = (table[ids[there].long()].float() * torch.tensor(scale, dtype=torch.float32)).to(table.dtype)      # one fp32 product, one rounding: the same bits
    assert torch.equal(out[1:n + 1], want)
    assert (out[0] == 7).all() and (out[n + 1] == 7).all()


def test_rows_copy_infinities_and_nan(torch_mod):
    torch = torch_mod
    table = torch.zeros((64, 64), dtype=torch.bfloat16, device="cuda")
    table[1], table[2], table[3] = float("nan"), float("inf"), float("-inf")
    ids = torch.tensor([3, -1, 1, 2, 64, 0], dtype=torch.int32, device="cuda")
    out = torch.full((6, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    with Model(64, 64, True) as (B, h):
        B.mace_embed_tokens(h, table, ids, out)
        B.mace_embed_tokens(h, table, ids[:0], out[:0])                     # no rows: nothing happens
        torch.cuda.synchronize()
    got = out.float().cpu()
    assert (got[0] == float("-inf")).all() and torch.isnan(got[2]).all() and (got[3] == float("inf")).all()
    assert (got[[1, 4, 5]] == 0).all()                                      # padding is zero, whatever the table holds


@pytest.mark.parametrize("bf16", [True, False])
def test_rows_unscaled_are_copies(torch_mod, bf16):
    """Every finite bit pattern of bf16, subnormal numbers and both zeros among them, and as many of fp32."""
    torch = torch_mod
    bits = torch.arange(65536, dtype=torch.int32, device="cuda")
    bits = bits[(bits & 0x7F80) != 0x7F80]
    bits = torch.cat([bits, bits[:(-len(bits)) % (64 * 64)]]).view(-1, 64)
    table = bits.to(torch.int16).view(torch.bfloat16) if bf16 else ((bits << 16) | (bits * 40503 & 0xFFFF)).view(torch.float32)
    n = table.shape[0]
    out = torch.empty_like(table)
    with Model(64, n, bf16) as (B, h):
        B.mace_embed_tokens(h, table, torch.arange(n, dtype=torch.int32, device="cuda"), out)
        torch.cuda.synchronize()
    kind = torch.int16 if bf16 else torch.int32
    assert torch.equal(out.view(kind), table.view(kind))


def check_grad(torch, d, vocab, ids, accumulate, scale, seed=0):
    n = ids.numel()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dx = torch.randn((n, d), generator=gen, device="cuda")
    there = (ids >= 0) & (ids < vocab)
    dx[~there] = float("nan")                                               # padding: never part of a sum
    old = torch.randn((vocab, d), generator=gen, device="cuda")
    got = old.clone() if accumulate else torch.full_like(old, float("nan"))
    again = got.clone()
    with Model(d, vocab, True) as (B, h):
        B.mace_embed_tokens_grad(h, ids, dx, got, workspace(torch, B, h, n), scale, accumulate)
        B.mace_embed_tokens_grad(h, ids, dx, again, workspace(torch, B, h, n + 1000), scale, accumulate)
        torch.cuda.synchronize()
    assert torch.equal(got, again)                                          # the order of the sums is that of the ids
    rows, v = dx[there].double() * scale, ids[there].long()
    base = old.double() if accumulate else torch.zeros_like(old, dtype=torch.float64)
    want = base.clone().index_add_(0, v, rows)
    # a sum of c terms (and the old value), each with one rounding of its product: at most c + 2 half steps of the sum of magnitudes
    count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, v, torch.ones_like(v, dtype=torch.float64))
    size = base.abs().index_add_(0, v, rows.abs())
    assert ((got.double() - want).abs() <= (count[:, None] + 2) * EPS32 * size).all()
    untouched = count == 0
    assert torch.equal(got[untouched], old[untouched] if accumulate else torch.zeros_like(old[untouched]))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind,n,d,vocab", [
    ("uniform", 1, 64, 64), ("uniform", 2, 128, 32000), ("one", 63, 64, 64), ("one", 65, 192, 128), ("two", 64, 256, 2048), ("padding", 100, 64, 640),
    ("text", 257, 256, 2048), ("uniform", 1000, 2048, 32000), ("sorted", 999, 1024, 512), ("runs", 4096, 320, 2048), ("text", 3347, 2048, 32000),
    ("one", 5000, 512, 1024), ("two", 4099, 4096, 6400), ("text", 20011, 1024, 128000), ("text", 2100, 8192, 704), ("uniform", 9000, 64, 64),
    ("text", 8192, 128, 32000), ("text", 8193, 128, 200000), ("uniform", 6001, 64, 200000)])
def test_grad(torch_mod, accumulate, kind, n, d, vocab):
    check_grad(torch_mod, d, vocab, draw_ids(torch_mod, kind, n, vocab, n), accumulate, 1.0 if n % 2 else 0.7)


def test_grad_long(torch_mod):
    """More rows than a step of the fine-tune-heavy configuration has, a third of them one token."""
    torch = torch_mod
    ids = draw_ids(torch, "text", 70001, 2048, 5)
    ids[::3] = 11
    check_grad(torch, 256, 2048, ids, True, 1.0)


@pytest.mark.parametrize("n", [700, 5000])
def test_grad_large_vocabulary(torch_mod, n):
    """More than 512 tokens to each of the 256 ranges in which the rows are sorted."""
    vocab = 262208
    ids = draw_ids(torch_mod, "text", n, vocab, n)
    ids[::7] = vocab - 1
    ids[1::7] = 0
    check_grad(torch_mod, 64, vocab, ids, n == 700, 1.0)


def test_grad_without_rows(torch_mod):
    torch = torch_mod
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    dx = torch.empty((0, 64), device="cuda")
    table = torch.full((128, 64), 3.0, device="cuda")
    with Model(64, 128, False) as (B, h):
        B.mace_embed_tokens_grad(h, none, dx, table, workspace(torch, B, h, 0), accumulate=True)
        torch.cuda.synchronize()
        assert (table == 3).all()
        B.mace_embed_tokens_grad(h, none, dx, table, workspace(torch, B, h, 0))
        torch.cuda.synchronize()
        assert (table == 0).all()


def test_grad_is_that_of_the_rows(torch_mod):
    """<dx, rows(E + u) - rows(E)> = <dE, u>: the rows are linear in the table.  Values are small integers, so every sum is exact."""
    torch = torch_mod
    d, vocab, n = 128, 320, 700
    gen = torch.Generator(device="cuda").manual_seed(3)
    small = lambda *s: torch.randint(-4, 5, s, generator=gen, device="cuda").float()
    E, u, dx = small(vocab, d), small(vocab, d), small(n, d)
    ids = draw_ids(torch, "text", n, vocab, 9)
    a, b, dE = torch.empty((n, d), device="cuda"), torch.empty((n, d), device="cuda"), torch.empty((vocab, d), device="cuda")
    with Model(d, vocab, False) as (B, h):
        B.mace_embed_tokens(h, E, ids, a, 2.0)
        B.mace_embed_tokens(h, E + u, ids, b, 2.0)
        B.mace_embed_tokens_grad(h, ids, dx, dE, workspace(torch, B, h, n), 2.0)
        torch.cuda.synchronize()
    assert (dx.double() * (b - a).double()).sum() == (dE.double() * u.double()).sum()


def test_graph_and_streams(torch_mod):
    """Captured on a side stream and replayed with new ids, eager calls in between: every replay gives the eager bits."""
    torch = torch_mod
    d, vocab, n = 512, 2048, 3001
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randn((vocab, d), generator=gen, device="cuda").to(torch.bfloat16)
    dx = torch.randn((n, d), generator=gen, device="cuda")
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    out, dE = torch.empty((n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((vocab, d), device="cuda")
    with Model(d, vocab, True) as (B, h):
        ws = workspace(torch, B, h, n)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            B.mace_embed_tokens(h, table, ids, out)
            B.mace_embed_tokens_grad(h, ids, dx, dE, ws)
        for turn in range(3):
            ids.copy_(draw_ids(torch, ("text", "one", "uniform")[turn], n, vocab, turn))
            want_out, want = torch.empty_like(out), torch.empty_like(dE)
            B.mace_embed_tokens(h, table, ids, want_out, stream=torch.cuda.current_stream())
            B.mace_embed_tokens_grad(h, ids, dx, want, workspace(torch, B, h, n))
            torch.cuda.synchronize()
            out.fill_(float("nan")); dE.fill_(float("nan")); ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want_out) and torch.equal(dE, want), turn


def test_binding_refuses_what_the_library_cannot_see(torch_mod):
    torch = torch_mod
    table = torch.zeros((128, 64), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(5, dtype=torch.int32, device="cuda")
    out = torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda")
    with Model(64, 128, True) as (B, h):
        for bad in (dict(table=table[:64]), dict(table=table.float()), dict(ids=ids.long()), dict(out=out[:4]), dict(out=out.float()), dict(ids=ids.cpu()),
                    dict(table=table.t().contiguous().t())):
            with pytest.raises(B.MaceError):
                B.mace_embed_tokens(h, bad.get("table", table), bad.get("ids", ids), bad.get("out", out))
        ws = workspace(torch, B, h, 5)
        dx, dE = torch.zeros((5, 64), device="cuda"), torch.zeros((128, 64), device="cuda")
        for bad in (dict(dx=dx[:4]), dict(dx=dx.to(torch.bfloat16)), dict(dE=dE[:64]), dict(ws=ws.cpu()), dict(ws=ws[:0])):
            with pytest.raises(B.MaceError):
                B.mace_embed_tokens_grad(h, ids, bad.get("dx", dx), bad.get("dE", dE), bad.get("ws", ws))
