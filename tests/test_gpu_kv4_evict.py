"""Eviction from the 4-bit paged cache through the C ABI against its definition: whole arrays, bit for bit."""
import numpy as np
import pytest

import kv4_reference as R
from test_gpu_kv4_cache import Model

pytestmark = pytest.mark.gpu


def workspace(torch, B, h, *sizes):
    return torch.full((B.mace_kv4_evict_workspace_bytes(h, *sizes),), 0xFF, dtype=torch.uint8, device="cuda")


def expected(cache, tables, lens, budgets, seq, n_sink, n_recent):
    """The pool's arrays behind the call, and the new lengths."""
    names = ("k", "v", "k_scale", "v_scale", "weight", "position")
    new = {n: getattr(cache, n).copy() for n in names}
    out = np.zeros((len(tables), cache.hkv), dtype=np.int32)
    for r, table in enumerate(tables):
        for h in range(cache.hkv):
            n = lens[r][h]
            t = np.arange(n)
            exists = (table[t // cache.size] >= 0) & (table[t // cache.size] < cache.blocks) if n else np.zeros(0, bool)
            at = lambda i: (table[i // cache.size], h, i % cache.size)
            w, p = np.zeros(n, np.float32), np.zeros(n, np.int64)
            w[exists], p[exists] = cache.weight[at(t[exists])], cache.position[at(t[exists])]
            keep = min(n, max(int(budgets[r][h]), 0))
            out[r, h] = keep
            if keep == n or keep == 0:
                continue
            stay = R.kept(w, p, exists, keep, n_sink, max(seq[r] - n_recent, 0) if n_recent else None)
            holes = sorted(set(range(keep)) - set(stay))
            moved = [i for i in stay if i >= keep]
            assert len(holes) == len(moved)
            for to, frm in zip(holes, moved):
                if exists[to] and exists[frm]:
                    for name in names:
                        new[name][at(to)] = getattr(cache, name)[at(frm)]
    return new, out


def run(torch, hkv, hd, size, lens, budgets, n_sink=0, n_recent=0, per_head=False, weights="random", seed=0, bad=(), max_context=None, in_place=False):
    r = np.random.default_rng(seed)
    with Model(hkv, hd, True) as (B, h):
        width = max([-(-l // size) for l in lens] + [1])
        cache = R.Cache(B, sum(-(-l // size) for l in lens) + 3, hkv, size, hd, seed)
        heads = [[int(r.integers(0, l + 1)) for _ in range(hkv)] if per_head else [l] * hkv for l in lens]
        tables = [cache.request(l, width) for l in lens]
        seq = [2 * l + 3 for l in lens]
        for table, l, sl in zip(tables, lens, seq):
            for hh in range(hkv):
                t = np.arange(l)
                at = (table[t // size], hh, t % size)
                cache.position[at] = r.permutation(sl)[:l]
                w = r.random(l).astype(np.float32) ** 6
                if weights == "ties":
                    w = r.integers(0, 3, l).astype(np.float32) / 4
                elif weights == "equal":
                    w[:] = 0.5
                elif weights == "odd":            # negative, NaN, infinite, subnormal, both zeros
                    w[r.random(l) < 0.5] = r.choice(np.array([np.nan, -1.0, np.inf, -np.inf, 1e-42, 0.0, -0.0, 3e38], np.float32))
                    w = np.where(r.random(l) < 0.3, r.choice(np.array([np.nan, -1.0, np.inf, 1e-42, -0.0], np.float32), l), w)
                cache.weight[at] = w
        for i, b in bad:
            tables[i][b] = [-1, cache.blocks, -2**31][b % 3]
        budgets = [[b] * hkv if np.isscalar(b) else list(b) for b in budgets]
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        mc = max(lens) if max_context is None else max_context
        d_lens = i32(heads) if per_head else i32(lens)
        new_lens = d_lens if in_place else torch.full((len(lens), hkv), -9, dtype=torch.int32, device="cuda")
        B.mace_kv4_evict(h, s, torch.from_numpy(np.stack(tables)).cuda(), d_lens, i32(seq), i32(budgets), new_lens, workspace(torch, B, h, len(lens), mc), mc, n_sink, n_recent)
        torch.cuda.synchronize()
        want, want_lens = expected(cache, tables, heads, budgets, seq, n_sink, n_recent)
        assert np.array_equal(new_lens.cpu().numpy(), want_lens)
        for name, x in want.items():
            got = cache.dev[name].cpu().numpy()
            assert np.array_equal(got.view(np.uint8), x.view(np.uint8)), name


@pytest.mark.parametrize("weights", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("hkv,hd,size,lens,budgets,n_sink,n_recent", [
    (2, 64, 16, [1, 2, 3, 40], [1, 1, 2, 0], 0, 0), (3, 128, 16, [100, 64, 65, 17], [50, 64, 1, 16], 4, 10), (1, 64, 1, [90], [33], 0, 5),
    (2, 128, 8, [500, 1023], [499, 512], 3, 600), (2, 64, 64, [1025, 2048, 0], [1024, 100, 5], 4, 128), (1, 128, 16, [2049, 2047], [1500, 2046], 0, 64)])
def test_against_the_definition(torch_mod, weights, hkv, hd, size, lens, budgets, n_sink, n_recent):
    run(torch_mod, hkv, hd, size, lens, budgets, n_sink, n_recent, weights=weights, seed=sum(lens))


@pytest.mark.parametrize("hd,lens,budgets", [(64, [4097, 4096], [2048, 4000]), (128, [9000], [8999]), (64, [32768], [7]), (128, [33000, 500], [20000, 499]), (64, [70001], [35000]),
                                             (128, [9000, 9000, 8200], [8700, 8000, 8193]), (64, [8193, 100], [7681, 99])])
def test_long_requests(torch_mod, hd, lens, budgets):
    """Around the lengths where keys no longer fit registers and the moves get a launch of their own."""
    run(torch_mod, 2, hd, 16, lens, budgets, 4, 100, seed=lens[0])
    run(torch_mod, 1, hd, 256, lens, budgets, 0, 0, weights="ties", seed=lens[0] + 1)


@pytest.mark.parametrize("in_place", [False, True])
def test_budgets_and_lengths_a_head(torch_mod, in_place):
    run(torch_mod, 4, 64, 16, [300, 77], [[10, 300, 0, 150], [76, -5, 1, 1000]], 2, 20, per_head=True, seed=3, in_place=in_place)
    run(torch_mod, 2, 128, 16, [5000, 10], [[10, 2500], [3, 9]], 2, 20, per_head=True, seed=4, in_place=in_place)


def test_more_protected_than_the_budget(torch_mod):
    run(torch_mod, 2, 64, 16, [200], [30], 100, 60, seed=5)             # the lowest positions first
    run(torch_mod, 2, 64, 16, [200], [30], 0, 300, seed=6)              # then the newest
    run(torch_mod, 2, 64, 16, [200], [30], 0, 10**9, seed=6)


def test_missing_blocks_and_bounds(torch_mod):
    run(torch_mod, 2, 64, 16, [200, 100], [120, 30], 4, 20, seed=7, bad=((0, 2), (0, 10), (1, 0)))
    # lengths above the bound are cut to it
    torch = torch_mod
    with Model(1, 64, True) as (B, h):
        cache = R.Cache(B, 20, 1, 16, 64, 0)
        table = cache.request(200, 13)
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        for given, bound in ((10**6, 100), (-4, 100), (10**6, 10**4)):
            cache.weight[:], cache.position[:] = cache.dev["weight"].cpu().numpy(), cache.dev["position"].cpu().numpy()
            cache.k[:], cache.v[:] = cache.dev["k"].cpu().numpy(), cache.dev["v"].cpu().numpy()
            cache.k_scale[:], cache.v_scale[:] = cache.dev["k_scale"].cpu().numpy(), cache.dev["v_scale"].cpu().numpy()
            new = i32([[-1]])
            B.mace_kv4_evict(h, s, torch.from_numpy(table[None]).cuda(), i32([given]), None, i32([[50]]), new, workspace(torch, B, h, 1, bound), bound)
            torch.cuda.synchronize()
            want, lens = expected(cache, [table], [[min(max(given, 0), bound, 13 * 16)]], [[50]], [0], 0, 0)
            assert np.array_equal(new.cpu().numpy(), lens)
            assert all(np.array_equal(cache.dev[k].cpu().numpy().view(np.uint8), x.view(np.uint8)) for k, x in want.items())


def test_captured_and_replayed(torch_mod):
    """Replayed with other budgets: every replay cuts what the one before it left."""
    torch = torch_mod
    hkv, hd, size = 2, 64, 16
    with Model(hkv, hd, True) as (B, h):
        cache = R.Cache(B, 400, hkv, size, hd, 1)
        tables = np.stack([cache.request(5000, 313)])
        cache.position[:] = np.random.default_rng(0).integers(0, 10**6, cache.position.shape)
        s = cache.upload(B)
        lens, budgets = (torch.full((1, hkv), 5000, dtype=torch.int32, device="cuda") for _ in range(2))
        ws, d_tab = workspace(torch, B, h, 1, 5000), torch.from_numpy(tables).cuda()
        call = lambda: B.mace_kv4_evict(h, s, d_tab, lens, None, budgets, lens, ws, 5000, n_sink=5)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for b in ([4000, 4999], [3999, 4999], [100, 2000], [100, 1]):
            for name in ("k", "v", "k_scale", "v_scale", "weight", "position"):
                getattr(cache, name)[:] = cache.dev[name].cpu().numpy()
            before = lens.tolist()
            budgets.copy_(torch.tensor([b]))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want, new = expected(cache, list(tables), before, [b], [0], 5, 0)
            assert np.array_equal(lens.cpu().numpy(), new)
            assert all(np.array_equal(cache.dev[k].cpu().numpy().view(np.uint8), x.view(np.uint8)) for k, x in want.items())
