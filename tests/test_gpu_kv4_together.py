"""The operators of long contexts on a compressed cache as a server uses them: a prompt, then decode steps of two requests whose heads are cut to budgets of
their own; every step is checked from what the one before it left on the device."""
import numpy as np
import pytest

import kv4_reference as R
from test_gpu_kv4_attention import check
from test_gpu_kv4_cache import Model
from test_gpu_kv4_evict import expected
from test_gpu_rotary import reference

pytestmark = pytest.mark.gpu


def test_prompt_decode_evict(torch_mod):
    torch = torch_mod
    from paper_2510_03283_amd import binding as B
    d, hkv, group, hd, size, rot = 512, 4, 2, 64, 16, 32
    hq = hkv * group
    cols, every = (hq + 2 * hkv) * hd, 6
    h = B.mace_create(d, hq, hkv, hd, 64, 64, 1e-6, 1e4, B.MACE_BF16)
    try:
        cache = R.Cache(B, 40, hkv, size, hd, 0)
        blocks = [[cache.free.pop() for _ in range(12)] for _ in range(2)]
        tables = np.array(blocks, dtype=np.int32)
        s = cache.upload(B)
        gen = torch.Generator().manual_seed(0)
        w = (torch.randn((cols, d), generator=gen) / 8).to(torch.bfloat16).cuda()
        freq = B.mace_rotary_frequencies(rot, 1e4, 4.0, 64)
        d_freq, d_tab = torch.from_numpy(freq).cuda(), torch.from_numpy(tables).cuda()
        budgets = np.stack([B.mace_kv_head_budget([1.0, 2.0, 3.0, 2.5], 4 * 60), B.mace_kv_head_budget([2.0, 2.0, 1.0, 1.0], 4 * 30)]).astype(np.int32)
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
        d_lens, d_budgets = i32(np.zeros((2, hkv))), i32(budgets)
        lens, seen = np.zeros((2, hkv), dtype=np.int64), [0, 0]
        mc = 190
        ws = torch.full((max(B.mace_kv4_attention_workspace_bytes(h, 2, 90, mc), B.mace_kv4_evict_workspace_bytes(h, 2, mc)),), 0xFF, dtype=torch.uint8, device="cuda")

        def pull():
            for name in ("k", "v", "k_scale", "v_scale", "weight", "position"):
                getattr(cache, name)[:] = cache.dev[name].cpu().numpy()

        for step in range(14):
            counts = [90, 41] if step == 0 else [1, 1]
            n = sum(counts)
            pos = np.concatenate([np.arange(a, a + c) for a, c in zip(seen, counts)]).astype(np.int32)
            x = torch.randn((n, d), generator=gen).to(torch.bfloat16).cuda()
            qkv = torch.empty((n, cols), dtype=torch.bfloat16, device="cuda")
            B.mace_gemm_bf16(h, 0, 0, n, cols, d, x, w, qkv)
            plain = qkv.clone()
            B.mace_rotary(h, qkv, i32(pos), d_freq, qkv, hq + hkv)                                 # queries and keys, in place; values stay
            q, k, v = qkv[:, :hq * hd], qkv[:, hq * hd:(hq + hkv) * hd], qkv[:, (hq + hkv) * hd:]
            slots = np.concatenate([np.stack([B.mace_kv_slot_mapping(tables[r], size, int(lens[r, hh]), counts[r]) for hh in range(hkv)], axis=1) for r in range(2)])
            pull()
            B.mace_kv4_append(h, s, k, v, i32(slots), i32(pos))
            torch.cuda.synchronize()
            want, sz = reference(plain.double().cpu().numpy(), pos, freq, hq + hkv, hd, False, 1.0, False)
            got = qkv.double().cpu().numpy()
            assert (np.abs(got[:, :want.shape[1]] - want) <= 4 * 2.0**-24 * sz + 2.0**-8 * np.abs(want) * (sz > 0)).all()
            assert torch.equal(v, plain[:, (hq + hkv) * hd:])
            for name, new in (("k", k), ("v", v)):
                code, scale = R.encode(new.double().cpu().numpy().reshape(n, hkv, hd))
                for hh in range(hkv):
                    at = (slots[:, hh] // size, hh, slots[:, hh] % size)
                    getattr(cache, name)[at], getattr(cache, name + "_scale")[at] = code[:, hh, 0::2] | code[:, hh, 1::2] << 4, scale[:, hh]
                    cache.weight[at], cache.position[at] = 0, pos
                assert np.array_equal(cache.dev[name].cpu().numpy(), getattr(cache, name)) and np.array_equal(cache.dev[name + "_scale"].cpu().numpy(), getattr(cache, name + "_scale"))
            assert np.array_equal(cache.dev["position"].cpu().numpy(), cache.position)

            before = cache.weight.copy()
            out, lse = torch.empty((n, hq * hd), dtype=torch.bfloat16, device="cuda"), torch.empty((n, hq), device="cuda")
            first = np.cumsum([0] + counts)
            B.mace_kv4_attention(h, s, q, d_tab, d_lens, out, ws, mc, q_offsets=i32(first) if step == 0 else None, max_rows=max(counts), lse=lse, add_weight=True)
            torch.cuda.synchronize()
            check(torch, True, cache, list(tables), lens.tolist(), list(zip(first[:-1].tolist(), counts)), q.cpu().reshape(n, hq, hd), out, lse, before, hd**-0.5)
            lens += np.array(counts)[:, None]
            seen = [a + c for a, c in zip(seen, counts)]
            d_lens.add_(i32(counts)[:, None])

            if step % every == 0:
                pull()
                B.mace_kv4_evict(h, s, d_tab, d_lens, i32(seen), d_budgets, d_lens, ws, mc, n_sink=2, n_recent=8)
                torch.cuda.synchronize()
                new, want_lens = expected(cache, list(tables), lens.tolist(), budgets, seen, 2, 8)
                assert np.array_equal(d_lens.cpu().numpy(), want_lens) and (want_lens < lens).any()
                assert all(np.array_equal(cache.dev[m].cpu().numpy().view(np.uint8), a.view(np.uint8)) for m, a in new.items())
                for r in range(2):                                          # the first tokens and the newest are still there
                    for hh in range(hkv):
                        t = np.arange(want_lens[r, hh])
                        held = set(new["position"][(tables[r][t // size], hh, t % size)].tolist())
                        assert {0, 1, *range(seen[r] - 8, seen[r])} <= held and len(held) == len(t)
                lens = want_lens.astype(np.int64)
    finally:
        B.mace_destroy(h)


def test_whole_cache_is_near_the_unrounded_attention(torch_mod):
    """Nothing evicted, values spread as a layer's: the 4-bit cache's attention against that of the rows before rounding, within what rounding to 4 bits can do.
    A value is off by at most 1/7 of its group's largest magnitude (half a step of 2 at 7 steps)."""
    torch = torch_mod
    from paper_2510_03283_amd import binding as B
    hkv, hd, n = 2, 128, 200
    h = B.mace_create(256, hkv, hkv, hd, 64, 64, 1e-6, 1e4, B.MACE_F32)
    try:
        gen = torch.Generator().manual_seed(0)
        k, v, q = (torch.randn((n, hkv * hd), generator=gen).cuda() for _ in range(3))
        cache = R.Cache(B, 13, hkv, 16, hd, 0, book=False)
        table = cache.request(0, 13)
        table[:] = np.random.default_rng(0).permutation(13)
        s = cache.upload(B)
        slots = torch.from_numpy(B.mace_kv_slot_mapping(table, 16, 0, n)).cuda()
        B.mace_kv4_append(h, s, k, v, slots)
        out = torch.empty_like(q)
        ws = torch.empty(B.mace_kv4_attention_workspace_bytes(h, 1, n, 0), dtype=torch.uint8, device="cuda")
        B.mace_kv4_attention(h, s, q, torch.from_numpy(table[None]).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"), out, ws, 0,
                             q_offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"), max_rows=n)
        torch.cuda.synchronize()
        qs, ks, vs = (x.double().cpu().view(n, hkv, hd).transpose(0, 1) for x in (q, k, v))
        x = (qs @ ks.transpose(1, 2) * hd**-0.5).masked_fill(torch.ones(n, n).triu(1).bool(), -np.inf)
        want = x.softmax(-1) @ vs
        off = lambda t: (t.abs().unflatten(-1, (-1, 32)).amax(-1) / 7).repeat_interleave(32, -1)     # bound of a value's error
        D = ((qs.abs() @ off(ks).transpose(1, 2)) * hd**-0.5).masked_fill(torch.ones(n, n).triu(1).bool(), 0).amax(-1, keepdim=True)
        bound = x.softmax(-1) @ off(vs) + (torch.exp(2 * D) - 1) * (x.softmax(-1) @ (vs.abs() + off(vs)))
        got = out.double().cpu().view(n, hkv, hd).transpose(0, 1)
        assert ((got - want).abs() <= bound + 1e-5).all()
    finally:
        B.mace_destroy(h)


def test_blocks_at_the_end_of_a_large_pool(torch_mod):
    """The same tokens in a small pool and in the last blocks of one whose byte offsets pass 2^32: attention, weights and eviction have the same bits."""
    torch = torch_mod
    hkv, hd, size, blocks, used = 8, 128, 16, 1 << 20, 24
    gen = torch.Generator().manual_seed(4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    x = torch.randn((used * size, hkv * hd), generator=gen).to(torch.bfloat16).cuda()
    order = torch.randperm(used, generator=gen)
    with Model(hkv, hd, True, 2) as (B, h):
        for count in (1, 20):                                           # few rows and many
            got = []
            for first, n in ((0, used), (blocks - used, blocks)):
                pool = lambda b, t=torch.uint8: torch.zeros((n, hkv, size, b) if b else (n, hkv, size), dtype=t, device="cuda")
                arrays = [pool(64), pool(64), pool(4), pool(4), pool(0, torch.float32), pool(0, torch.int32)]
                s = B.kv4_cache_struct(*arrays)
                slots = (first + order[torch.arange(used * size) // size]) * size + torch.arange(used * size) % size
                B.mace_kv4_append(h, s, x, x.flip(0).contiguous(), slots.int().cuda(), positions=i32(list(range(used * size))))
                table, lens = (first + order).int().cuda().view(1, used), i32([used * size - count])
                q = torch.randn((count, 2 * hkv * hd), generator=torch.Generator().manual_seed(count)).to(torch.bfloat16).cuda()
                out, work = torch.empty_like(q), lambda b: torch.empty(b, dtype=torch.uint8, device="cuda")
                B.mace_kv4_attention(h, s, q, table, lens, out, work(B.mace_kv4_attention_workspace_bytes(h, 1, count, used * size)), used * size, q_offsets=i32([0, count]),
                                     max_rows=count, add_weight=True)
                new = torch.empty((1, hkv), dtype=torch.int32, device="cuda")
                B.mace_kv4_evict(h, s, table, i32([used * size]), i32([used * size]), i32([[100] * hkv]), new, work(B.mace_kv4_evict_workspace_bytes(h, 1, used * size)), used * size, 4, 16)
                torch.cuda.synchronize()
                got.append([out.clone()] + [a[first:].clone() for a in arrays])
                del arrays, s
            assert (got[0][0] != 0).any() and (got[0][5] > 0).any()
            assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("max_rows,group,bf16", [(1, 1, True), (3, 4, False), (40, 2, True), (300, 4, True), (40, 2, False)])
def test_nothing_behind_the_workspace_is_written(torch_mod, max_rows, group, bf16):
    """Requests of all sizes up to the bounds, in a workspace of exactly the stated size and in one with bytes of every kind before the call: the same outputs, and the bytes behind stay."""
    torch = torch_mod
    hkv, hd, size, mc = 2, 64, 16, 5000
    r = np.random.default_rng(max_rows)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()
    with Model(hkv, hd, bf16, group) as (B, h):
        n_req = 5
        counts, lens = np.array([max_rows, 1, max_rows // 2, 0, max_rows]), np.array([mc, mc, 300, 70, 0])
        cache = R.Cache(B, 700, hkv, size, hd, 1)
        tables = np.stack([cache.request(int(l + c), -(-(mc + max_rows) // size)) for l, c in zip(lens, counts)])
        s = cache.upload(B)
        first = np.concatenate([[0], np.cumsum(counts)])
        dtype = torch.bfloat16 if bf16 else torch.float32
        q = torch.from_numpy(r.standard_normal((int(first[-1]), hkv * group * hd)).astype(np.float32)).to(dtype).cuda()
        kept = {n: cache.dev[n].clone() for n in cache.dev}
        results = []
        for fill, budget in ((0x00, 1000), (0xFF, 1000), (0x7F, 1000)):
            for n in kept:
                cache.dev[n].copy_(kept[n])
            size_a, size_e = B.mace_kv4_attention_workspace_bytes(h, n_req, max_rows, mc), B.mace_kv4_evict_workspace_bytes(h, n_req, mc)
            wa, we = (torch.full((b + 4096,), fill, dtype=torch.uint8, device="cuda") for b in (size_a, size_e))
            out, lse = torch.empty_like(q), torch.empty((q.shape[0], hkv * group), device="cuda")
            B.mace_kv4_attention(h, s, q, i32(tables), i32(lens), out, wa[:size_a], mc, q_offsets=i32(first), max_rows=max_rows, lse=lse, add_weight=True)
            new = torch.empty((n_req, hkv), dtype=torch.int32, device="cuda")
            B.mace_kv4_evict(h, s, i32(tables), i32(lens), i32(lens), i32(np.full((n_req, hkv), budget)), new, we[:size_e], mc, 4, 16)
            torch.cuda.synchronize()
            assert (wa[size_a:] == fill).all() and (we[size_e:] == fill).all()
            results.append([out, lse, new] + [cache.dev[n].view(torch.uint8).clone() for n in kept])
        for other in results[1:]:
            assert all(torch.equal(a.view(torch.uint8) if a.dtype != torch.int32 else a, b.view(torch.uint8) if b.dtype != torch.int32 else b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("mc", [1, 63, 64, 65, 1000, 8193])
def test_lists_of_the_eviction_fit_their_workspace(torch_mod, mc):
    """Every token of the first half goes, every one behind it stays: the longest lists that there are."""
    torch = torch_mod
    hkv, hd, size = 2, 64, 16
    with Model(hkv, hd, True) as (B, h):
        cache = R.Cache(B, 2 * (mc // size + 1), hkv, size, hd, 3)
        table = np.stack([cache.request(mc, mc // size + 1) for _ in range(2)])
        t = np.arange(mc)
        for r in range(2):
            for hh in range(hkv):
                cache.weight[table[r][t // size], hh, t % size] = t
        s = cache.upload(B)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        need = B.mace_kv4_evict_workspace_bytes(h, 2, mc)
        work = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
        new = torch.empty((2, hkv), dtype=torch.int32, device="cuda")
        keep = (mc + 1) // 2
        B.mace_kv4_evict(h, s, torch.from_numpy(table).cuda(), i32([mc, mc]), i32([mc, mc]), i32([[keep] * hkv] * 2), new, work[:need], mc)
        torch.cuda.synchronize()
        assert (work[need:] == 0xAB).all() and (new == keep).all()
        got = cache.dev["weight"].cpu().numpy()
        for r in range(2):
            for hh in range(hkv):
                assert sorted(got[table[r][t // size], hh, t % size][:keep]) == list(range(mc - keep, mc))


def test_scales_at_four_byte_alignment(torch_mod):
    """k_scale, v_scale, weight and position may begin at any multiple of four bytes."""
    torch = torch_mod
    hkv, size = 2, 16
    for hd in (64, 128):
        with Model(hkv, hd, True, 4) as (B, h):
            cache = R.Cache(B, 40, hkv, size, hd, 2)
            table = cache.request(400, 25)[None]
            s = cache.upload(B)
            q = torch.randn((1, hkv * 4 * hd), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()

            def go(s, count):
                rows = q.repeat(count, 1)
                out = torch.empty_like(rows)
                work = torch.empty(B.mace_kv4_attention_workspace_bytes(h, 1, count, 400), dtype=torch.uint8, device="cuda")
                B.mace_kv4_attention(h, s, rows, torch.from_numpy(table).cuda(), torch.tensor([400 - count], dtype=torch.int32, device="cuda"), out, work, 400,
                                     q_offsets=torch.tensor([0, count], dtype=torch.int32, device="cuda"), max_rows=count, add_weight=True)
                torch.cuda.synchronize()
                return out

            moved = {}
            for n in ("k_scale", "v_scale", "weight", "position"):
                raw = cache.dev[n].view(torch.uint8).flatten()
                moved[n] = torch.empty(raw.numel() + 4, dtype=torch.uint8, device="cuda")[4:]
                moved[n].copy_(raw)
                moved[n] = moved[n].view(cache.dev[n].dtype).view(cache.dev[n].shape)
                assert moved[n].data_ptr() % 16 == 4
            s2 = B.kv4_cache_struct(cache.dev["k"], cache.dev["v"], moved["k_scale"], moved["v_scale"], moved["weight"], moved["position"])
            for count in (1, 5, 60):
                assert torch.equal(go(s, count), go(s2, count))
            assert torch.equal(moved["weight"].view(torch.uint8), cache.dev["weight"].view(torch.uint8))


class Step:
    """One step of a server on buffers of its own: rotary, append behind the cached tokens, attention with weights, eviction."""

    def __init__(self, torch, B, h, hd, seed, rows, max_rows):
        self.torch, self.B, self.h, self.max_rows = torch, B, h, max_rows
        hkv, group, size, mc = 2, 4, 16, 3000
        gen = torch.Generator().manual_seed(seed)
        cache = self.cache = R.Cache(B, 600, hkv, size, hd, seed)
        self.tables_host = [cache.request(mc + max_rows, -(-(mc + max_rows) // size)) for _ in range(3)]
        self.tables = torch.from_numpy(np.stack(self.tables_host)).cuda()
        self.s = cache.upload(B)
        self.start = {n: x.clone() for n, x in cache.dev.items()}
        self.x = torch.randn((rows, (group + 2) * hkv * hd), generator=gen).to(torch.bfloat16).cuda()
        self.y = torch.empty((rows, (group + 1) * hkv * hd), dtype=torch.bfloat16, device="cuda")
        self.freq = torch.from_numpy(B.mace_rotary_frequencies(hd // 2, 1e4, 4.0, 2048)).cuda()
        self.positions, self.slots = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        self.offsets, self.lens, self.total = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 3, 3))
        self.budgets = torch.full((3, hkv), 900, dtype=torch.int32, device="cuda")
        self.new = torch.empty((3, hkv), dtype=torch.int32, device="cuda")
        self.out = torch.empty((rows, group * hkv * hd), dtype=torch.bfloat16, device="cuda")
        self.mc, self.q_cols, self.kv_cols = mc, group * hkv * hd, hkv * hd
        self.work = torch.empty(B.mace_kv4_attention_workspace_bytes(h, 3, max_rows, mc), dtype=torch.uint8, device="cuda")
        self.work2 = torch.empty(B.mace_kv4_evict_workspace_bytes(h, 3, mc + max_rows), dtype=torch.uint8, device="cuda")

    def fill(self, lens, counts):
        torch = self.torch
        first = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        positions, slots = np.zeros(len(self.slots), np.int32), np.full(len(self.slots), -1, np.int32)
        for table, l, c, f in zip(self.tables_host, lens, counts, first):
            t = l + np.arange(c)
            positions[f:f + c], slots[f:f + c] = t, table[t // 16] * 16 + t % 16
        put = lambda to, x: to.copy_(torch.from_numpy(np.asarray(x, dtype=np.int32)))
        put(self.positions, positions), put(self.slots, slots), put(self.offsets, first), put(self.lens, lens), put(self.total, np.add(lens, counts))
        for n, x in self.start.items():
            self.cache.dev[n].copy_(x)
        self.out.zero_()

    def run(self):
        B, h = self.B, self.h
        B.mace_rotary(h, self.x[:, :self.q_cols + self.kv_cols], self.positions, self.freq, self.y, (self.q_cols + self.kv_cols) // self.h.head_dim)
        B.mace_kv4_append(h, self.s, self.y[:, self.q_cols:], self.x[:, self.q_cols + self.kv_cols:], self.slots, positions=self.positions)
        B.mace_kv4_attention(h, self.s, self.y[:, :self.q_cols], self.tables, self.lens, self.out, self.work, self.mc, q_offsets=self.offsets, max_rows=self.max_rows, add_weight=True)
        B.mace_kv4_evict(h, self.s, self.tables, self.total, self.total, self.budgets, self.new, self.work2, self.mc + self.max_rows, 4, 64)

    def result(self):
        self.torch.cuda.synchronize()
        return [self.out.clone(), self.new.clone()] + [x.view(self.torch.uint8).clone() for x in self.cache.dev.values()]


SIZES = [([900, 20, 2999], [1, 1, 1]), ([0, 2500, 63], [2, 1, 0]), ([3000, 3000, 3000], [2, 2, 2]), ([5, 0, 1], [0, 2, 1])]


@pytest.mark.parametrize("hd,max_rows", [(64, 2), (128, 2), (128, 60)])
def test_a_captured_step_is_replayed_with_other_lengths(torch_mod, hd, max_rows):
    torch = torch_mod
    sizes = [(l, [c * max_rows // 2 for c in n]) for l, n in SIZES]
    with Model(2, hd, True, 4) as (B, h):
        step, want = Step(torch, B, h, hd, 1, 3 * max_rows, max_rows), []
        for l, n in sizes:
            step.fill(l, n)
            step.run()
            want.append(step.result())
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                step.run()
        for turn in range(3):
            for i in range(len(sizes)):
                step.fill(*sizes[(i + turn) % len(sizes)])
                graph.replay()
                assert all(torch.equal(a, b) for a, b in zip(step.result(), want[(i + turn) % len(sizes)]))


def test_two_servers_on_two_streams(torch_mod):
    """Handles, pools and workspaces of their own: what two streams do at the same time does not meet."""
    torch = torch_mod
    with Model(2, 128, True, 4) as (B, h), Model(2, 64, True, 4) as (_, h2):
        steps = [Step(torch, B, h, 128, 1, 180, 60), Step(torch, B, h2, 64, 2, 6, 2)]
        sizes = [SIZES[0][0], SIZES[2][0]], [[60, 3, 59], [1, 2, 2]]
        want = []
        for step, l, n in zip(steps, *sizes):
            step.fill(l, n)
            step.run()
            want.append(step.result())
        streams = [torch.cuda.Stream() for _ in steps]
        for _ in range(5):
            for step, l, n in zip(steps, *sizes):
                step.fill(l, n)
            torch.cuda.synchronize()
            for step, stream in zip(steps, streams):
                with torch.cuda.stream(stream):
                    step.run()
            torch.cuda.synchronize()
            for step, w in zip(steps, want):
                assert all(torch.equal(a, b) for a, b in zip(step.result(), w))
