"""Attention over the 4-bit paged cache through the C ABI against its definition in 64 bits."""
import numpy as np
import pytest

import kv4_reference as R
from test_gpu_kv4_cache import Model

pytestmark = pytest.mark.gpu


def workspace(torch, B, h, *sizes):
    return torch.full((B.mace_kv4_attention_workspace_bytes(h, *sizes),), 0xFF, dtype=torch.uint8, device="cuda")


def check(torch, bf16, cache, tables, lens, rows, q, out, lse, before, scale, weight=True, margin=1):
    """Bounds: D = rounding of a product of hd terms in fp32 (hd + 2 half steps of the sum of magnitudes) is an error of the exponent; exponentials and sums add
    half steps of fp32, one a token at most; bf16 probabilities half a step of bf16 (2^-8), and so does the output."""
    hd = q.shape[2]
    want, want_lse, absv, bound, w = R.attention(cache, tables, lens, rows, q.double().cpu().numpy(), scale)
    live = [f + i for f, c in rows for i in range(c)]
    most = max([max(l) + c for l, (_, c) in zip(lens, rows)] + [1])
    D = (hd + 2) * 2.0**-24 * bound[..., 0] + 2.0**-24 * (16 + 6 * bound[..., 1])
    rel = 2 * D + most * 2.0**-24
    got, got_lse = out.double().cpu().numpy().reshape(want.shape), lse.double().cpu().numpy()
    tol = absv * rel[..., None] + (2.0**-8 * (absv * 1.01 + np.abs(want)) if bf16 else 2.0**-23 * absv) + 1e-30
    err = np.abs(got - want)
    assert (err[live] <= tol[live]).all(), (err[live] / tol[live]).max()
    finite = np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(got_lse[live]), ~finite[live])
    with np.errstate(invalid="ignore"):
        assert (np.abs(got_lse - want_lse)[live] <= (rel + 2.0**-23 * np.abs(want_lse))[live])[finite[live]].all()
    if weight:
        now = cache.dev["weight"].double().cpu().numpy()
        expect, slack = before.astype(np.float64).copy(), np.zeros_like(before, dtype=np.float64)
        group = q.shape[1] // cache.hkv
        for table, got_w, (f, c) in zip(tables, w, rows):
            for hh, x in enumerate(got_w):
                t = np.arange(len(x))
                there = (table[t // cache.size] >= 0) & (table[t // cache.size] < cache.blocks) if len(t) else t.astype(bool)
                t = t[there]
                if not len(t) or not c:
                    continue
                at = (table[t // cache.size], hh, t % cache.size)
                np.add.at(expect, at, x[there])
                np.add.at(slack, at, x[there] * (rel[f:f + c, hh * group:(hh + 1) * group].max() + (c * group + 8) * 2.0**-24) + 1e-36)
        slack += 4 * 2.0**-24 * np.abs(expect)
        assert np.array_equal(np.isnan(now), np.isnan(expect))
        with np.errstate(invalid="ignore"):
            assert (np.abs(now - expect) <= slack)[~np.isnan(expect)].all(), np.nanmax(np.abs(now - expect) / slack)


def run(torch, bf16, hkv, group, hd, size, lens, counts, offsets=True, per_head=False, gap=0, scale=None, wide=False, spread=1.0, seed=0, add_weight=True, extra=0, ld=0, most=1, bound=0):
    """One call: requests of lens[r] cached tokens and counts[r] new rows; `gap` rows in front and behind that belong to nobody."""
    r = np.random.default_rng(seed)
    dtype = torch.bfloat16 if bf16 else torch.float32
    with Model(hkv, hd, bf16, group) as (B, h):
        width = max([-(-(l + c) // size) for l, c in zip(lens, counts)] + [1]) + extra
        cache = R.Cache(B, sum(-(-(l + c) // size) for l, c in zip(lens, counts)) + 2, hkv, size, hd, seed, wide=wide)
        heads = [[int(r.integers(0, l + 1)) for _ in range(hkv)] if per_head else [l] * hkv for l in lens]
        tables = [cache.request(l + c, width, [x + c for x in hl]) for l, c, hl in zip(lens, counts, heads)]
        first = np.cumsum([gap] + counts)
        rows = [(int(f), c) for f, c in zip(first, counts)]
        n, hq = int(first[-1]) + gap, hkv * group
        s = cache.upload(B)
        before = cache.weight.copy()
        q = torch.from_numpy((spread * r.standard_normal((n, hq * hd + ld))).astype(np.float32)).to(dtype)
        out = torch.full((n, hq * hd + 2 * ld), 5.0, dtype=dtype, device="cuda")
        lse = torch.full((n, hq), 5.0, device="cuda")
        d_lens = torch.tensor(heads if per_head else lens, dtype=torch.int32, device="cuda")
        d_off = torch.from_numpy(first.astype(np.int32)).cuda() if offsets else None
        d_tab = torch.from_numpy(np.stack(tables)).cuda()
        mc, mr = max(lens + [bound]), max(counts + [most])
        sizes = (len(lens), mr, mc)
        B.mace_kv4_attention(h, s, q.cuda(), d_tab, d_lens, out, workspace(torch, B, h, *sizes), mc, q_offsets=d_off, max_rows=mr, lse=lse, scale=scale, add_weight=add_weight)
        torch.cuda.synchronize()
        live = [f + i for f, c in rows for i in range(c)]
        dead = [i for i in range(n) if i not in set(live)]
        assert (out[dead] == 5).all() and (lse[dead] == 5).all() and (out[:, hq * hd:] == 5).all()
        assert torch.equal(cache.dev["position"].cpu(), torch.from_numpy(cache.position)) and torch.equal(cache.dev["k"].cpu(), torch.from_numpy(cache.k))
        check(torch, bf16, cache, tables, heads, rows, q[:, :hq * hd].view(n, hq, hd), out[:, :hq * hd].contiguous(), lse, before, hd**-0.5 if scale is None else scale, add_weight)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hkv,group,hd,size,lens", [
    (1, 1, 64, 16, [0]), (2, 1, 128, 16, [0, 1, 15, 16, 17, 63, 64, 65]), (1, 8, 128, 16, [255, 256, 257, 300]), (2, 4, 64, 32, [1000, 3, 511, 0]),
    (3, 2, 64, 1, [70, 5]), (2, 8, 64, 2, [129, 31]), (1, 4, 128, 8, [333, 64]), (1, 2, 128, 4, [190]), (1, 1, 128, 256, [255, 256, 700]), (1, 4, 64, 128, [4100, 4095])])
def test_one_row_a_request(torch_mod, bf16, hkv, group, hd, size, lens):
    run(torch_mod, bf16, hkv, group, hd, size, lens, [1] * len(lens), offsets=False, seed=sum(lens) + hd, ld=8)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hkv,group,hd,size,lens,counts,gap", [
    (2, 1, 64, 16, [0, 5, 40], [1, 17, 3], 0), (1, 4, 128, 16, [100, 0, 250], [5, 33, 1], 2), (2, 8, 64, 16, [63, 64, 65], [2, 2, 2], 0), (1, 1, 128, 16, [0], [150], 1),
    (1, 2, 64, 8, [300, 20, 7, 1], [0, 40, 0, 9], 0), (1, 8, 128, 64, [600], [37], 3), (1, 1, 64, 16, [1500, 3], [1, 70], 0),
    (1, 1, 128, 16, [2100, 5], [130, 3], 0), (2, 2, 64, 4, [1100], [65], 0), (1, 4, 64, 32, [0, 1, 62], [64, 32, 90], 0)])
def test_several_rows_a_request(torch_mod, bf16, hkv, group, hd, size, lens, counts, gap):
    run(torch_mod, bf16, hkv, group, hd, size, lens, counts, gap=gap, seed=sum(lens) + sum(counts))


@pytest.mark.parametrize("hkv,group,hd,lens,counts,per_head", [
    (1, 8, 128, [5000], [17], False), (1, 4, 64, [9000, 3], [15, 40], False),             # rows that many thread blocks work on
    (2, 4, 128, [0, 700, 64, 1300, 5, 0, 2000], [33, 5, 0, 200, 1, 0, 70], True), (3, 1, 128, [300, 0, 100], [130, 260, 1], True),
    (1, 2, 64, [63, 64, 65, 127, 128, 129], [64, 64, 64, 65, 63, 128], False)])
@pytest.mark.parametrize("shares", [True, False])
def test_rows_cut_into_shares(torch_mod, hkv, group, hd, lens, counts, per_head, shares):
    """Shares where the bounds promise work enough, else equal splits of blocks of rows."""
    run(torch_mod, True, hkv, group, hd, 16, lens, counts, per_head=per_head, gap=1, seed=sum(lens), bound=64 * 24 * 512 if shares else 0)


@pytest.mark.parametrize("hd", [64, 128])
def test_more_requests_than_threads(torch_mod, hd):
    r = np.random.default_rng(hd)
    lens, counts = [int(x) for x in r.integers(0, 60, 600)], [int(x) for x in r.integers(0, 4, 600)]
    counts[17], lens[400] = 60, 900
    run(torch_mod, True, 1, 2, hd, 16, lens, counts, seed=1, bound=4000)


@pytest.mark.parametrize("hd", [64, 128])
def test_blocks_of_rows_in_a_grid(torch_mod, hd):
    r = np.random.default_rng(hd)
    lens, counts = [int(x) for x in r.integers(0, 300, 64)], [int(x) for x in r.integers(0, 20, 64)]
    run(torch_mod, True, 1, 8, hd, 16, lens, counts, seed=2, most=256)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hd,group", [(64, 4), (128, 1), (128, 4)])
def test_heads_of_different_length(torch_mod, bf16, hd, group):
    run(torch_mod, bf16, 4, group, hd, 16, [200, 77, 900], [1, 1, 1], offsets=False, per_head=True, seed=hd + group)
    run(torch_mod, bf16, 4, group, hd, 16, [200, 77], [6, 20], per_head=True, seed=hd + group + 1)


@pytest.mark.parametrize("bf16", [True, False])
def test_scales_of_the_products(torch_mod, bf16):
    """A negative one, none, and sharp rows over values of very different size."""
    for scale, spread, wide in ((-0.2, 1.0, False), (0.0, 1.0, False), (0.125, 30.0, False), (2.0**-9, 1.0, True)):
        run(torch_mod, bf16, 2, 4, 64, 16, [300, 65], [1, 1], offsets=False, scale=scale, spread=spread, wide=wide, seed=7)
        run(torch_mod, bf16, 1, 2, 128, 16, [150], [11], scale=scale, spread=spread, wide=wide, seed=8)


def test_tables_longer_than_needed_and_no_weights(torch_mod):
    run(torch_mod, True, 2, 2, 64, 16, [100, 30], [1, 1], offsets=False, extra=9, add_weight=False, seed=3)


@pytest.mark.parametrize("bf16", [True, False])
def test_missing_blocks_and_rows_without_a_token(torch_mod, bf16):
    """Entries outside the cache are left out; a request without any block has out 0 and lse -inf; lengths that the table has no room for are cut."""
    torch = torch_mod
    hkv, group, hd, size = 2, 4, 64, 16
    dtype = torch.bfloat16 if bf16 else torch.float32
    with Model(hkv, hd, bf16, group) as (B, h):
        cache = R.Cache(B, 60, hkv, size, hd, 5)
        a, b = cache.request(301, 20), cache.request(20, 20)
        a[3], a[7], a[18] = -1, 60, 2**31 - 1
        none = np.full(20, -5, dtype=np.int32)
        s = cache.upload(B)
        before = cache.weight.copy()
        lens = [300, 19, 40]
        q = torch.randn((3, 8 * hd), generator=torch.Generator().manual_seed(1)).to(dtype)
        out, lse = torch.full((3, 8 * hd), 5.0, dtype=dtype, device="cuda"), torch.full((3, 8), 5.0, device="cuda")
        t = torch.from_numpy(np.stack([a, b, none])).cuda()
        B.mace_kv4_attention(h, s, q.cuda(), t, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, workspace(torch, B, h, 3, 1, 400), 400, lse=lse, add_weight=True)
        torch.cuda.synchronize()
        assert (out[2] == 0).all() and torch.isneginf(lse[2]).all()
        check(torch, bf16, cache, [a, b, none], [[l] * hkv for l in lens], [(i, 1) for i in range(3)], q.view(3, 8, hd), out, lse, before, hd**-0.5)
        # a table of 2 blocks for lengths of 5000 and -3: 32 tokens and 1
        out2 = torch.empty_like(out[:2])
        B.mace_kv4_attention(h, s, q[:2].cuda(), t[:2, :2].contiguous(), torch.tensor([5000, -3], dtype=torch.int32, device="cuda"), out2, workspace(torch, B, h, 2, 1, 400), 400,
                             lse=lse[:2])
        torch.cuda.synchronize()
        check(torch, bf16, cache, [a[:2], b[:2]], [[31] * hkv, [0] * hkv], [(0, 1), (1, 1)], q[:2].view(2, 8, hd), out2, lse[:2], before, hd**-0.5, weight=False)
        # more rows than the table has places: the first ones see nothing
        q3 = torch.randn((40, 8 * hd), generator=torch.Generator().manual_seed(2)).to(dtype)
        out3, lse3 = torch.empty((40, 8 * hd), dtype=dtype, device="cuda"), torch.empty((40, 8), device="cuda")
        off = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
        B.mace_kv4_attention(h, s, q3.cuda(), t[:1, :2].contiguous(), torch.tensor([0], dtype=torch.int32, device="cuda"), out3, workspace(torch, B, h, 1, 40, 0), 0,
                             q_offsets=off, max_rows=40, lse=lse3)
        torch.cuda.synchronize()
        assert (out3[:8] == 0).all() and torch.isneginf(lse3[:8]).all() and torch.isfinite(lse3[8:]).all()


@pytest.mark.parametrize("hd,count", [(128, 6), (128, 40), (64, 70)])
def test_nan_stays_where_it_is_attended_to(torch_mod, hd, count):
    """A NaN key makes NaN the rows that see it, a NaN value their 32 columns, a NaN query its own row; the other rows keep their bits."""
    torch = torch_mod
    hkv, group, size = 2, 2, 16
    with Model(hkv, hd, True, group) as (B, h):
        cache = R.Cache(B, 30, hkv, size, hd, 9)
        tables = np.stack([cache.request(80 + count, 10), cache.request(70, 10)])
        s = cache.upload(B)
        n, see = count + 4, 3                                           # rows 3 .. count - 1 of request 0 see token 83
        q = torch.randn((n, 4 * hd), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        off = torch.tensor([0, count, n], dtype=torch.int32, device="cuda")
        lens = torch.tensor([80, 60], dtype=torch.int32, device="cuda")

        def go():
            out = torch.empty_like(q)
            B.mace_kv4_attention(h, s, q, torch.from_numpy(tables).cuda(), lens, out, workspace(torch, B, h, 2, count, 80), 80, q_offsets=off, max_rows=count)
            torch.cuda.synchronize()
            return out.view(n, 4, hd)

        clean = go()
        at = (int(tables[0, 83 // 16]), 1, 83 % 16)
        codes, old = cache.dev["v"][at][16:32].clone(), int(cache.dev["v_scale"][at][1])
        cache.dev["v_scale"][at][1], cache.dev["v"][at][16:32] = 255, 0       # as the append leaves it
        got = go()
        assert torch.isnan(got[see:count, 2:, 32:64]).all()
        got[see:count, 2:, 32:64] = clean[see:count, 2:, 32:64]
        assert torch.equal(got, clean)
        cache.dev["v_scale"][at][1], cache.dev["v"][at][16:32] = old, codes
        old = int(cache.dev["k_scale"][at][0])
        cache.dev["k_scale"][at][0] = 255
        got = go()
        assert torch.isnan(got[see:count, 2:]).all()
        got[see:count, 2:] = clean[see:count, 2:]
        assert torch.equal(got, clean)
        cache.dev["k_scale"][at][0] = old
        q[count + 1, :hd] = float("nan")
        got = go()
        assert torch.isnan(got[count + 1, 0]).all()
        got[count + 1, 0] = clean[count + 1, 0]
        assert torch.equal(got, clean)


def test_shared_blocks(torch_mod):
    """Requests below one prefix list the same leading blocks: their weights get both requests' probabilities."""
    torch = torch_mod
    hkv, group, hd, size = 2, 2, 64, 16
    with Model(hkv, hd, True, group) as (B, h):
        cache = R.Cache(B, 40, hkv, size, hd, 2)
        a, b = cache.request(150, 12), cache.request(150, 12)
        b[:4] = a[:4]
        s = cache.upload(B)
        before = cache.weight.copy()
        lens = [149, 120]
        q = torch.randn((2, 4 * hd), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
        out, lse = torch.empty((2, 4 * hd), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 4), device="cuda")
        B.mace_kv4_attention(h, s, q.cuda(), torch.from_numpy(np.stack([a, b])).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out,
                             workspace(torch, B, h, 2, 1, 149), 149, lse=lse, add_weight=True)
        torch.cuda.synchronize()
        check(torch, True, cache, [a, b], [[l] * hkv for l in lens], [(0, 1), (1, 1)], q.view(2, 4, hd), out, lse, before, hd**-0.5)


def test_the_same_call_gives_the_same_bits(torch_mod):
    torch = torch_mod
    hkv, group, hd, size = 4, 4, 128, 16
    with Model(hkv, hd, True, group) as (B, h):
        cache = R.Cache(B, 700, hkv, size, hd, 4)
        lens = [3000, 1, 4097, 900]
        tables = torch.from_numpy(np.stack([cache.request(l + 1, 257) for l in lens])).cuda()
        s = cache.upload(B)
        w0 = cache.dev["weight"].clone()
        q = torch.randn((4, 16 * hd), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        d_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        first = None
        for _ in range(3):
            cache.dev["weight"].copy_(w0)
            out, lse = torch.empty_like(q), torch.empty((4, 16), device="cuda")
            B.mace_kv4_attention(h, s, q, tables, d_lens, out, workspace(torch, B, h, 4, 1, 4097), 4097, lse=lse, add_weight=True)
            torch.cuda.synchronize()
            now = (out.view(torch.int16), lse.view(torch.int32), cache.dev["weight"].view(torch.int32).clone())
            assert first is None or all(torch.equal(x, y) for x, y in zip(now, first))
            first = now


def test_captured_and_replayed_with_other_lengths(torch_mod):
    """A captured decode call is replayed with lengths and queries written over in between; on a side stream."""
    torch = torch_mod
    hkv, group, hd, size = 2, 4, 64, 16
    with Model(hkv, hd, True, group) as (B, h):
        cache = R.Cache(B, 200, hkv, size, hd, 6)
        tables = [cache.request(1100, 80) for _ in range(2)]
        s = cache.upload(B)
        q = torch.zeros((2, 8 * hd), dtype=torch.bfloat16, device="cuda")
        lens = torch.zeros(2, dtype=torch.int32, device="cuda")
        out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")
        ws, d_tab = workspace(torch, B, h, 2, 1, 1099), torch.from_numpy(np.stack(tables)).cuda()
        call = lambda: B.mace_kv4_attention(h, s, q, d_tab, lens, out, ws, 1099, lse=lse, add_weight=True)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for step, ll in enumerate(([0, 5], [1099, 300], [64, 1000], [2, 2])):
            q.copy_(torch.randn((2, 8 * hd), generator=torch.Generator().manual_seed(step)))
            lens.copy_(torch.tensor(ll))
            torch.cuda.synchronize()
            before = cache.dev["weight"].cpu().numpy()
            graph.replay()
            torch.cuda.synchronize()
            check(torch, True, cache, tables, [[l] * hkv for l in ll], [(0, 1), (1, 1)], q.cpu().view(2, 8, hd), out, lse, before, hd**-0.5)
