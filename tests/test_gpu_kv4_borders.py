"""Attention over the 4-bit paged cache and eviction from it at the borders of what their documentation says: errors, NaN, infinities, missing blocks."""
import numpy as np
import pytest

import kv4_reference as R
from test_gpu_kv4_attention import run as attention_run, workspace
from test_gpu_kv4_cache import Model
from test_gpu_kv4_evict import expected as evicted, workspace as evict_workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hkv,group,hd,lens,counts,spread", [
    (2, 1, 128, [300, 1000], [1, 1], 1.0), (2, 4, 128, [700, 64], [1, 1], 1.0), (2, 8, 128, [900], [1], 1.0), (2, 4, 64, [500, 1300], [1, 1], 1.0), (1, 2, 64, [800], [8], 1.0),
    (2, 2, 128, [600, 90], [40, 3], 1.0), (1, 4, 64, [1000], [20], 1.0), (1, 8, 128, [2500, 30], [33, 70], 1.0), (1, 4, 128, [400], [60], 20.0), (1, 2, 128, [400], [1], 20.0)])
def test_bf16_rows_err_by_their_outputs_rounding(torch_mod, hkv, group, hd, lens, counts, spread):
    """Half a step of the output (2^-8 of it) and, of every token's part of it, 2^-16 for its probability and the fp32 bounds: D, an error of the exponent, from a product of hd
    terms (hd + 2 half steps of fp32 of the sum of magnitudes) and 16 + 6 |x| half steps in the exponential, twice (numerator and sum), and a half step a token in the sums."""
    torch, size = torch_mod, 16
    r = np.random.default_rng(sum(lens) + group)
    with Model(hkv, hd, True, group) as (B, h):
        cache = R.Cache(B, sum(-(-(l + c) // size) for l, c in zip(lens, counts)) + 2, hkv, size, hd, 3)
        width = max(-(-(l + c) // size) for l, c in zip(lens, counts))
        tables = [cache.request(l + c, width) for l, c in zip(lens, counts)]
        s = cache.upload(B)
        n, hq = sum(counts), hkv * group
        q = torch.from_numpy((spread * r.standard_normal((n, hq * hd))).astype(np.float32)).to(torch.bfloat16)
        first = np.cumsum([0] + counts)
        out = torch.empty((n, hq * hd), dtype=torch.bfloat16, device="cuda")
        B.mace_kv4_attention(h, s, q.cuda(), torch.from_numpy(np.stack(tables)).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out,
                             workspace(torch, B, h, len(lens), max(counts), max(lens)), max(lens), q_offsets=torch.from_numpy(first.astype(np.int32)).cuda(), max_rows=max(counts))
        torch.cuda.synchronize()
        want, _, absv, bound, _ = R.attention(cache, tables, [[l] * hkv for l in lens], list(zip(first, counts)), q.double().numpy().reshape(n, hq, hd), hd**-0.5)
        most = max(l + c for l, c in zip(lens, counts))
        D = (hd + 2) * 2.0**-24 * bound[..., 0] + 2.0**-24 * (16 + 6 * bound[..., 1])
        part = (2.0**-16 + 2 * D + most * 2.0**-24)[..., None] * absv
        err = np.abs(out.double().cpu().numpy().reshape(want.shape) - want)
        tol = 2.0**-8 * np.abs(want) + 1.01 * part + 1e-30
        assert (err <= tol).all(), (err / tol).max()


def weights_of(cache, table, head, tokens):
    """Bits of the weights of a request's first tokens."""
    t = np.arange(tokens)
    return cache.dev["weight"].cpu().numpy()[table[t // cache.size], head, t % cache.size].view(np.uint32)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hd,count", [(128, 6), (64, 8), (128, 9), (128, 40), (64, 70), (128, 150)])
def test_weights_are_nan_only_where_a_nan_row_attends(torch_mod, bf16, hd, count):
    """Of few and of many rows: a NaN query makes NaN the weights of the tokens up to its own, a NaN key those of its head, a NaN value none; all others keep the bits of a clean call."""
    torch = torch_mod
    hkv, group, size, ctx = 2, 2, 16, 80
    dtype = torch.bfloat16 if bf16 else torch.float32
    with Model(hkv, hd, bf16, group) as (B, h):
        cache = R.Cache(B, 30, hkv, size, hd, 9)
        tables = [cache.request(ctx + count, 15), cache.request(70, 15)]
        s = cache.upload(B)
        w0 = cache.dev["weight"].clone()
        n = count + 4
        q = torch.randn((n, 4 * hd), generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
        off, lens = torch.tensor([0, count, n], dtype=torch.int32, device="cuda"), torch.tensor([ctx, 60], dtype=torch.int32, device="cuda")
        d_tab = torch.from_numpy(np.stack(tables)).cuda()

        def go():
            cache.dev["weight"].copy_(w0)
            B.mace_kv4_attention(h, s, q, d_tab, lens, torch.empty_like(q), workspace(torch, B, h, 2, count, ctx), ctx, q_offsets=off, max_rows=count, add_weight=True)
            torch.cuda.synchronize()
            return [weights_of(cache, tables[0], hh, ctx + count) for hh in range(hkv)] + [weights_of(cache, tables[1], hh, 64) for hh in range(hkv)]

        def same(got, but=()):
            return all(np.array_equal(g, c) for k, (g, c) in enumerate(zip(got, clean)) if k not in but)

        clean = go()
        assert not any(np.isnan(c.view(np.float32)).any() for c in clean)
        for row in (0, 1, count - 2, count - 1):
            old = q[row, hd:2 * hd].clone()
            q[row, hd:2 * hd] = float("nan")                  # query head 1, so kv head 0
            got = go()
            q[row, hd:2 * hd] = old
            assert np.isnan(got[0].view(np.float32)[:ctx + row + 1]).all() and np.array_equal(got[0][ctx + row + 1:], clean[0][ctx + row + 1:]) and same(got, (0,))
        at = (int(tables[0][83 // size]), 1, 83 % size)
        for name, spread in (("v_scale", ()), ("k_scale", (1,))):
            old = int(cache.dev[name][at][0])
            cache.dev[name][at][0] = 255
            got = go()
            cache.dev[name][at][0] = old
            assert same(got, spread) and all(np.isnan(got[k].view(np.float32)).all() for k in spread)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hd,count", [(128, 2), (64, 6), (128, 40), (64, 70)])
def test_products_that_are_all_minus_infinity(torch_mod, bf16, hd, count):
    """Such a row is one without a token: out 0, lse -inf, and weights that keep their bits."""
    torch = torch_mod
    hkv, group, size, ctx = 1, 2, 16, 200
    dtype = torch.bfloat16 if bf16 else torch.float32
    with Model(hkv, hd, bf16, group) as (B, h):
        cache = R.Cache(B, 20, hkv, size, hd, 4)
        table = cache.request(ctx + count, 20)
        cache.k[:] = 0xEE                                     # every key -4 steps (code 14)
        s = cache.upload(B)
        before = weights_of(cache, table, 0, ctx + count)
        q = torch.full((count, group * hd), 3e38, dtype=dtype, device="cuda")
        off, lens = torch.tensor([0, count], dtype=torch.int32, device="cuda"), torch.tensor([ctx], dtype=torch.int32, device="cuda")
        out, lse = torch.full_like(q, 5.0), torch.full((count, group), 5.0, device="cuda")
        B.mace_kv4_attention(h, s, q, torch.from_numpy(table[None]).cuda(), lens, out, workspace(torch, B, h, 1, count, ctx), ctx, q_offsets=off, max_rows=count, lse=lse, scale=1.0,
                             add_weight=True)
        torch.cuda.synchronize()
        assert (out == 0).all() and torch.isneginf(lse).all()
        assert np.array_equal(weights_of(cache, table, 0, ctx + count), before)


def test_eviction_into_a_missing_block(torch_mod):
    """By hand: of tokens 0, 1 (no block), 2, 3 the two of largest weight stay, token 2 at place 0; token 3 would move to place 1, which there is none of, and stays behind the new length."""
    torch = torch_mod
    with Model(1, 64, True) as (B, h):
        cache = R.Cache(B, 8, 1, 1, 64, 3)
        table = cache.request(4, 4)
        cache.weight[table] = np.float32([0.25, 0.75, 0.5, 1.0]).reshape(4, 1, 1)
        names = ("k", "v", "k_scale", "v_scale", "weight", "position")
        want = {n: getattr(cache, n).copy() for n in names}
        for n in names:
            want[n][table[0]] = want[n][table[2]]
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        new = i32([[-1]])
        ws = torch.full((B.mace_kv4_evict_workspace_bytes(h, 1, 4),), 0xFF, dtype=torch.uint8, device="cuda")
        B.mace_kv4_evict(h, s, i32([[table[0], 8, table[2], table[3]]]), i32([4]), None, i32([[2]]), new, ws, 4)
        torch.cuda.synchronize()
        assert new.tolist() == [[2]]
        assert all(np.array_equal(cache.dev[n].cpu().numpy().view(np.uint8), x.view(np.uint8)) for n, x in want.items())


@pytest.mark.parametrize("top", [100, 2**30 - 1])
def test_sinks_rank_above_the_newest_up_to_the_last_position(torch_mod, top):
    """Two tokens, the newest in front of a sink, one place: the sink takes it."""
    torch = torch_mod
    with Model(1, 64, True) as (B, h):
        cache = R.Cache(B, 4, 1, 1, 64, 3)
        table = cache.request(2, 2)
        cache.position[table] = np.int32([top, top - 1]).reshape(2, 1, 1)
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        new = i32([[-1]])
        ws = torch.full((B.mace_kv4_evict_workspace_bytes(h, 1, 2),), 0xFF, dtype=torch.uint8, device="cuda")
        B.mace_kv4_evict(h, s, i32([list(table)]), i32([2]), i32([top + 1]), i32([[1]]), new, ws, 2, n_sink=top, n_recent=1)
        torch.cuda.synchronize()
        assert new.tolist() == [[1]] and int(cache.dev["position"][int(table[0])]) == top - 1


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("hkv,group,hd,lens,counts", [
    (1, 1, 128, [1024, 1000], [1, 1]), (2, 4, 64, [2048, 1025, 1024, 1023], [1, 1, 1, 1]), (1, 2, 128, [2047, 1026], [1, 1]), (1, 1, 64, [1024, 960], [16, 16]), (1, 1, 64, [1024], [64]),
    (1, 1, 64, [1024], [65]), (1, 1, 64, [1086, 1088], [2, 1]), (8, 1, 64, [1024 * 32, 1024 * 31 + 5], [3, 1])])
def test_the_last_split_takes_a_tail(torch_mod, bf16, hkv, group, hd, lens, counts):
    """Splits of 1024 tokens: lengths with the rows' own tokens on both sides of what the last of them takes, 64 more (the last case: 32 splits in a full chip)."""
    attention_run(torch_mod, bf16, hkv, group, hd, 16, lens, counts, seed=sum(lens))


@pytest.mark.parametrize("bf16", [True, False])
def test_one_row_of_a_matrix_of_any_width(torch_mod, bf16):
    """A single row has no stride: its matrix may be wider than the heads by any number of columns, in every operator that takes rows."""
    torch = torch_mod
    hkv, group, hd, size = 2, 2, 64, 16
    dtype = torch.bfloat16 if bf16 else torch.float32
    with Model(hkv, hd, bf16, group) as (B, h):
        cache = R.Cache(B, 4, hkv, size, hd, 1)
        table = cache.request(20, 2)
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        x = torch.randn((1, 4 * hd + 3), generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
        narrow, wide = (torch.full((1, 4 * hd + w), 5.0, dtype=dtype, device="cuda") for w in (0, 1))
        freq = torch.from_numpy(B.mace_rotary_frequencies(hd, 1e4)).cuda()
        slot = i32([int(table[1]) * size + 4])
        for out, rows in ((narrow, x[:, :4 * hd].contiguous()), (wide, x)):
            B.mace_rotary(h, rows, i32([20]), freq, out, 4)
            B.mace_kv4_append(h, s, rows, rows, slot, i32([20]))
            kept = [cache.dev[n].clone() for n in ("k", "v", "k_scale", "v_scale")]
            turned = out.clone()
            B.mace_kv4_attention(h, s, rows, i32([list(table)]), i32([20]), out, workspace(torch, B, h, 1, 1, 20), 20)
            torch.cuda.synchronize()
            if out is narrow:
                first = kept, turned, out.clone()
            else:
                assert all(torch.equal(a, b) for a, b in zip(kept, first[0]))
                assert torch.equal(turned[:, :-1], first[1]) and torch.equal(out[:, :-1], first[2]) and (out[:, -1] == 5).all()


@pytest.mark.parametrize("hd,bound,tokens,moves", [
    (64, 8192, [8192, 8191], [600, 513]), (128, 8193, [8193, 8193, 8192], [511, 512, 513]), (64, 9000, [9000, 9000], [513, 512]), (128, 9000, [8900], [4000]),
    (64, 32768, [32768, 32767], [512, 513]), (128, 32769, [32769, 32768], [513, 512]), (64, 32769, [5], [2])])
def test_evictions_at_the_limits_of_their_kernels(torch_mod, hd, bound, tokens, moves):
    """Bounds up to 8192 move everything in the selecting block, longer ones up to 512 tokens a head there and more in a launch of their own; up to 32768 keys stay in LDS.  Exactly
    `moves` tokens of head 0 are displaced, fewer of head 1."""
    torch, hkv, size = torch_mod, 2, 16
    r = np.random.default_rng(bound + hd)
    with Model(hkv, hd, True) as (B, h):
        cache = R.Cache(B, sum(-(-t // size) for t in tokens) + 1, hkv, size, hd, 1)
        width = -(-bound // size)
        tables, budgets = [cache.request(t, width) for t in tokens], []
        for table, n, m in zip(tables, tokens, moves):
            keep = n - max(m, n // 3) if n > 5 else 3
            budgets.append([keep] * hkv)
            for head, k in ((0, m), (1, m // 2)):
                w = r.random(n).astype(np.float32) / 4 + 1       # of those behind the new length only k stay, in the places of k in front of it
                w[keep:] /= 8
                w[r.choice(keep, k, replace=False)] /= 16
                w[keep + r.choice(n - keep, k, replace=False)] += 2
                t = np.arange(n)
                cache.weight[table[t // size], head, t % size] = w
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        new = i32([[-1] * hkv] * len(tokens))
        B.mace_kv4_evict(h, s, torch.from_numpy(np.stack(tables)).cuda(), i32(tokens), None, i32(budgets), new, evict_workspace(torch, B, h, len(tokens), bound), bound)
        torch.cuda.synchronize()
        want, lens = evicted(cache, tables, [[t] * hkv for t in tokens], budgets, tokens, 0, 0)
        assert np.array_equal(new.cpu().numpy(), lens)
        for table, m, (keep, _) in zip(tables, moves, budgets):
            t = np.arange(keep)
            at = (table[t // size], 0, t % size)
            assert (want["position"][at] != cache.position[at]).sum() == m
        for name, x in want.items():
            assert np.array_equal(cache.dev[name].cpu().numpy().view(np.uint8), x.view(np.uint8)), name


@pytest.mark.parametrize("hd,count", [(128, 1), (64, 8), (128, 30)])
def test_the_largest_fp32_queries_stay_finite(torch_mod, hd, count):
    """Between the largest bf16 number and the largest fp32 one, against keys that are 0 there: as with 0 in their place, bit for bit."""
    torch = torch_mod
    hkv, group, size, ctx = 1, 2, 16, 100
    with Model(hkv, hd, False, group) as (B, h):
        cache = R.Cache(B, 20, hkv, size, hd, 4)
        table = cache.request(ctx + count, 20)
        cache.k[..., 3] &= 0xF0                               # element 6 of every key
        s = cache.upload(B)
        w0 = cache.dev["weight"].clone()
        q = torch.randn((count, group * hd), generator=torch.Generator().manual_seed(1)).cuda()
        off, lens = torch.tensor([0, count], dtype=torch.int32, device="cuda"), torch.tensor([ctx], dtype=torch.int32, device="cuda")
        got = []
        for x in (0.0, 3.4e38, -3.4028234663852886e38):
            q[:, 6::hd] = x
            cache.dev["weight"].copy_(w0)
            out = torch.empty_like(q)
            B.mace_kv4_attention(h, s, q, torch.from_numpy(table[None]).cuda(), lens, out, workspace(torch, B, h, 1, count, ctx), ctx, q_offsets=off, max_rows=count, add_weight=True)
            torch.cuda.synchronize()
            got.append((out.view(torch.int32).clone(), weights_of(cache, table, 0, ctx + count)))
        assert torch.isfinite(got[0][0].view(torch.float32)).all()
        assert all(torch.equal(g[0], got[0][0]) and np.array_equal(g[1], got[0][1]) for g in got[1:])
