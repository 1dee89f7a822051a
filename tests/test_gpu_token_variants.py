"""The variants of the operators at the two ends of a model that only large calls take (inputs or outputs that the last-level cache cannot
hold, many short rows), the smallest calls with banned tokens, and what lies behind the workspace."""
import math

import pytest

import test_gpu_embed as embed
import test_gpu_token_logprobs as logprobs
from test_gpu_token_logprobs import EPS, INF, lib  # noqa: F401

pytestmark = pytest.mark.gpu
GUARD = 4096
LLC = 256 << 20


@pytest.fixture(autouse=True)
def guarded(torch_mod, monkeypatch):
    """Every workspace has exactly the bytes that were asked for, and bytes behind them that must not change."""
    torch = torch_mod
    made = []

    def padded(need):
        buf = torch.full((need + GUARD,), 0xFF, dtype=torch.uint8, device="cuda")
        buf[need:] = 0xA5
        made.append(buf)
        return buf[:need]

    monkeypatch.setattr(logprobs, "workspace", lambda torch, lib, n, vocab, k: padded(lib[0].mace_token_logprobs_workspace_bytes(lib[1], n, vocab, k)))
    monkeypatch.setattr(embed, "workspace", lambda torch, B, h, n: padded(B.mace_embed_grad_workspace_bytes(h, n)))
    yield
    torch.cuda.synchronize()
    for buf in made:
        assert (buf[-GUARD:] == 0xA5).all(), buf.numel() - GUARD


# ---- many short rows: a wave each, several turns
def check_wave_rows(torch, x, token, o, k):
    """Rows (fp32 or bf16, without NaN or +inf) that one wave each sums: at most vocab / 64 additions a thread, a rescaling a turn and a tree
    of six, which is below vocab / 64 + 32; twice that, as each addition may meet a factor of its own."""
    n, vocab = x.shape
    x64 = x.double()
    m = x64.max(dim=1, keepdim=True).values
    empty = torch.isneginf(m)
    t = torch.where(torch.isneginf(x64), -INF, x64 - torch.where(empty, 0.0, m))
    e = t.exp()
    s = torch.where(empty, 1.0, e.sum(dim=1, keepdim=True))
    L = s.log()
    far = torch.where(e > 0, -t, 0.0)                               # the distance to the maximum of every column that counts
    mean, mean2 = (e * far).sum(dim=1, keepdim=True) / s, (e * far * far).sum(dim=1, keepdim=True) / s
    depth = 2 * (vocab / 64 + 32)
    # e^t: 3 |t| half steps of t and its product with log2 e, 4 of the exponential; L: as much as the sum, and its own logarithm's
    rel = EPS * (3 * mean + depth + 4)
    tol_L = rel + EPS * (4 + 2 * L)
    got_m, got_L = o["row_stats"][:, :1].double(), o["row_stats"][:, 1:].double()
    assert torch.equal(got_m, m) and ((got_L - L).abs() <= tol_L).all()

    def close(got, columns, given):
        want = torch.where(given, torch.where(empty, -INF, t - L).gather(1, columns), 0.0)
        fin = torch.isfinite(want)
        assert torch.equal(got[~fin], want[~fin])
        slack = tol_L + EPS * 2 * (far.gather(1, columns) + L + 1)
        assert ((got - want).abs() <= slack)[fin].all()

    given = (token >= 0) & (token < vocab)
    close(o["logp"].double()[:, None], token.clamp(0, vocab - 1).long()[:, None], given[:, None])
    H = torch.where(empty, 0.0, L + mean)
    tol_H = tol_L + EPS * (3 * mean2 + (depth + 8) * mean) + mean * rel + EPS * 4 * H
    assert ((o["entropy"].double()[:, None] - H).abs() <= torch.where(empty, 0.0, tol_H)).all()
    if k:
        order = x.float().sort(dim=1, descending=True, stable=True)
        ids, gone = order.indices[:, :k], torch.isneginf(order.values[:, :k])
        assert torch.equal(o["top_ids"].long(), torch.where(gone, -1, ids))
        got = o["top_logp"].double()
        assert (got[gone] == -INF).all()
        close(torch.where(gone, 0.0, got), ids, ~gone)


WAVE_ROWS = [(2048, 8192), (2100, 8191), (2500, 4099), (3000, 1025)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,vocab", WAVE_ROWS)
def test_a_wave_a_row(torch_mod, lib, dtype, n, vocab):  # noqa: F811
    """One to eight turns of a wave; more columns at the threshold than candidates fit (lowest, equal, coarse)."""
    torch = torch_mod
    for kind, k in (("peaked", 0), ("plain", 20), ("banned", 32), ("lowest", 20), ("equal", 32), ("coarse", 32), ("rising", 20), ("falling", 1)):
        print(kind, k, flush=True)
        x, token = logprobs.draw(torch, n, vocab, kind, n + k)
        rows = logprobs.rows_of(torch, x, vocab + vocab % 2, 1 if kind == "plain" else 0, dtype)
        o = logprobs.call(torch, lib, rows, token, k)
        torch.cuda.synchronize()
        check_wave_rows(torch, rows, token, o, k)


# ---- inputs and outputs past the last-level cache.  n, vocab, row stride, first element, type
WAVE_ROWS_PAST = [(8200, 8192, 8192, 0, "fp32"), (16500, 8191, 8192, 0, "bf16")]
ROWS_PAST = [(2200, 32000, 32000, 0, "fp32"), (1400, 50001, 50001, 0, "fp32"), (1100, 128011, 128064, 0, "bf16"), (1100, 128011, 128011, 1, "bf16")]


def size(dtype):
    return 4 if dtype == "fp32" else 2


@pytest.mark.parametrize("n,vocab,ld,offset,dtype", WAVE_ROWS_PAST + ROWS_PAST)
def test_logits_past_the_cache(torch_mod, lib, n, vocab, ld, offset, dtype):  # noqa: F811
    torch = torch_mod
    assert n * vocab * size(dtype) > LLC
    for kind, k in (("peaked", 0), ("banned", 8), ("lowest", 32)):
        print(kind, k, flush=True)
        x, token = logprobs.draw(torch, n, vocab, kind, n + k)
        rows = logprobs.rows_of(torch, x, ld, offset, dtype)
        del x
        o = logprobs.call(torch, lib, rows, token, k)
        # without the entropy other kernels run: the same bits
        names = ["logp", "row_stats"] + (["top_ids", "top_logp"] if k else [])
        part = {key: torch.full_like(o[key], 77) for key in names}
        lib[0].mace_token_logprobs(lib[1], rows, logprobs.workspace(torch, lib, n, vocab, k), token, **part)
        torch.cuda.synchronize()
        assert all(torch.equal(part[key], o[key]) for key in names)
        if (n, vocab, ld, offset, dtype) in ROWS_PAST:
            logprobs.check(torch, rows, token, o, k)
            continue
        for r0 in range(0, n, 2100):                                          # in slices: the reference is in 64 bits
            r = slice(r0, min(n, r0 + 2100))
            check_wave_rows(torch, rows[r], token[r], {key: None if v is None else v[r] for key, v in o.items()}, k)


GRADS_PAST = [(2200, 32000, "fp32", 0), (2200, 32000, "fp32", 1), (4400, 32000, "bf16", 0), (4400, 32000, "bf16", 1)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,vocab,out,odd", GRADS_PAST)
def test_gradient_past_the_cache(torch_mod, lib, dtype, n, vocab, out, odd):  # noqa: F811
    torch = torch_mod
    assert n * vocab * size(out) > LLC
    x, token = logprobs.draw(torch, n, vocab, "banned", n)
    rows = logprobs.rows_of(torch, x, vocab + odd, odd, dtype)
    del x
    logprobs.grad_check(torch, lib, rows, token, dtype, out, True, True, vocab + odd)
    if dtype == out:
        logprobs.grad_check(torch, lib, rows, token, dtype, out, False, True, in_place=True)


EMBED_PAST = [(17000, 4096, True), (9000, 4096, False)]


@pytest.mark.parametrize("n,d,bf16", EMBED_PAST)
def test_rows_past_the_cache(torch_mod, n, d, bf16):
    assert 2 * n * d * (2 if bf16 else 4) >= LLC
    embed.test_rows(torch_mod, bf16, n, d, 640, 64.0)
    embed.test_rows(torch_mod, bf16, n, d, 32000, 1.0)


# rows, width, vocabulary: the rows' gradients past half the cache; the table held by it or not
TABLE_PAST = [(9000, 4096, 12800), (9000, 4096, 32000)]
FEW_PAST = [(100, 4096, 32000), (0, 4096, 32000)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,d,vocab", TABLE_PAST + FEW_PAST)
def test_table_gradient_past_the_cache(torch_mod, accumulate, n, d, vocab):
    assert 8 * n * d >= LLC or 4 * vocab * d > LLC
    embed.check_grad(torch_mod, d, vocab, embed.draw_ids(torch_mod, "text", n, vocab, n), accumulate, 0.7)


# ---- what lies behind the workspace
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(1, 32000), (1, 65505), (1, 65536), (3, 128011), (2, 131072), (7, 262145), (64, 128011), (170, 98304), (255, 66000), (511, 140001), (600, 131073)])
def test_nothing_is_written_behind_the_workspace(torch_mod, lib, dtype, n, vocab):  # noqa: F811
    """Rows that several blocks share, around the sizes where their number changes."""
    torch = torch_mod
    x, token = logprobs.draw(torch, n, vocab, "plain", n)
    for ld, offset, k in ((vocab + -vocab % 64, 0, 32), (vocab + 1, 1, 0), (vocab, 63, 1)):
        rows = logprobs.rows_of(torch, x, ld, offset, dtype)
        o = logprobs.call(torch, lib, rows, token, k)
        torch.cuda.synchronize()
        logprobs.check(torch, rows, token, o, k)


@pytest.mark.parametrize("n,d,vocab", [(257, 64, 64), (300, 8192, 640), (1024, 256, 2048), (4096, 1024, 2048), (4097, 64, 2048), (8192, 64, 2048), (8193, 2048, 2048), (16385, 128, 300032)])
def test_nothing_is_written_behind_the_gradients_workspace(torch_mod, n, d, vocab):
    for kind in ("one", "text", "runs"):                                      # all sums, some and few set aside
        embed.check_grad(torch_mod, d, vocab, embed.draw_ids(torch_mod, kind, n, vocab, n), kind == "text", 1.0)


# ---- one and two rows with banned tokens
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 700, 8193, 32000, 128011])
@pytest.mark.parametrize("n", [1, 2])
def test_one_request_held_to_a_grammar(torch_mod, lib, dtype, n, vocab):  # noqa: F811
    """Most tokens banned, all but one, all; the given token allowed and banned."""
    torch = torch_mod
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    base, token = logprobs.draw(torch, n, vocab, "plain", vocab)
    for allowed in ("some", "one", "none"):
        x = base.clone()
        if allowed == "some":
            x[torch.rand((n, vocab), generator=gen, device="cuda") < 0.9] = -INF
        else:
            x[:] = -INF
            if allowed == "one":
                x[:, vocab // 2] = base[:, vocab // 2]
        if n == 2:
            x[1] = base[1]                                                    # the other request is free
        rows = logprobs.rows_of(torch, x, vocab, 0, dtype)
        for at in (vocab // 2, 0, -1):
            token[:] = at
            for k in (0, 5, 32):
                o = logprobs.call(torch, lib, rows, token, k)
                torch.cuda.synchronize()
                logprobs.check(torch, rows, token, o, k)
                if allowed == "one" and at == vocab // 2:
                    assert o["logp"][0] == 0 and o["entropy"][0] == 0
                elif allowed == "none" and at >= 0:
                    assert o["logp"][0] == -math.inf and o["entropy"][0] == 0
            logprobs.grad_check(torch, lib, rows, token, dtype, dtype, True, True)
