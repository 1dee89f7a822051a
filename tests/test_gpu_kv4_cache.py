"""The 4-bit paged cache through the C ABI: rounding, scatter by slot, reading back, bit for bit."""
import numpy as np
import pytest

import kv4_reference as R

pytestmark = pytest.mark.gpu


class Model:
    def __init__(self, hkv, hd, bf16, group=1):
        from paper_2510_03283_amd import binding as B
        self.B, self.h = B, B.mace_create(256, hkv * group, hkv, hd, 64, 64, 1e-6, 1e4, B.MACE_BF16 if bf16 else B.MACE_F32)

    def __enter__(self):
        return self.B, self.h

    def __exit__(self, *_):
        self.B.mace_destroy(self.h)


def inputs(torch, kind, n, cols, seed, dtype):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((n, cols), generator=gen)
    if kind == "wide":                   # groups from the smallest to the largest numbers, subnormal ones among them
        x *= torch.exp2(torch.randint(-148, 126, (n, cols // 32, 1), generator=gen).float()).expand(-1, -1, 32).reshape(n, cols)
        x[0] = 0.0
        x[-1, ::3] = -0.0
    elif kind == "borders":              # halves, ties and the limits of a step
        x = torch.randint(-64, 65, (n, cols), generator=gen).float() / 8.0
        x[:, ::32] = torch.tensor([4.0, 6.0, 7.0, 7.0625, 7.9375])[torch.randint(0, 5, (n, cols // 32), generator=gen)]
    elif kind == "bad":                  # groups with a NaN or an infinity
        x.view(-1)[torch.randperm(n * cols, generator=gen)[:n]] = float("nan")
        x.view(-1)[torch.randperm(n * cols, generator=gen)[:n]] = float("inf")
        x.view(-1)[torch.randperm(n * cols, generator=gen)[:n]] = float("-inf")
    return x.to(dtype)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,hkv,hd,size,kind,per_head,pad", [(1, 1, 64, 1, "wide", False, 0), (1, 4, 128, 16, "wide", True, 8), (33, 4, 64, 16, "borders", False, 64),
                                                             (70, 8, 128, 2, "bad", True, 0), (517, 3, 64, 256, "wide", False, 16), (1000, 2, 128, 8, "borders", True, 0)])
def test_append_and_gather(torch_mod, bf16, n, hkv, hd, size, kind, per_head, pad):
    torch = torch_mod
    dtype = torch.bfloat16 if bf16 else torch.float32
    cols, blocks = hkv * hd, -(-n // size) + 3
    k, v = (inputs(torch, kind, n, cols + pad, s, dtype) if kind != "wide" or pad % 32 == 0 else inputs(torch, kind, n, cols + 32, s, dtype)[:, :cols + pad].contiguous()
            for s in (n, n + 1))
    with Model(hkv, hd, bf16) as (B, h):
        cache = R.Cache(B, blocks, hkv, size, hd, n)
        s = cache.upload(B)
        r = np.random.default_rng(n)
        slots = np.stack([r.permutation(blocks * size)[:n] for _ in range(hkv)], axis=1) if per_head else r.permutation(blocks * size)[:n]
        slots = slots.astype(np.int32)
        stored = r.random(slots.shape) >= 0.1
        slots[~stored] = r.choice([-1, blocks * size, 2**31 - 1, -2**31], (~stored).sum())
        positions = r.integers(0, 2**30, n).astype(np.int32)
        ko, vo = (torch.full((n, cols), 3.0, dtype=dtype, device="cuda") for _ in range(2))
        d_slots = torch.from_numpy(slots).cuda()
        B.mace_kv4_append(h, s, k.cuda(), v.cuda(), d_slots, torch.from_numpy(positions).cuda())
        B.mace_kv4_gather(h, s, d_slots, ko, vo)
        torch.cuda.synchronize()
        # the pool as the definition leaves it
        where, ok = (slots, stored) if per_head else (np.repeat(slots[:, None], hkv, 1), np.repeat(stored[:, None], hkv, 1))
        row, head = np.nonzero(ok)
        slot = where[row, head]
        at = (slot // size, head, slot % size)
        for x, name, out in ((k, "k", ko), (v, "v", vo)):
            code, scale = R.encode(x[:, :cols].double().numpy().reshape(n, hkv, hd))
            codes = getattr(cache, name).copy()
            codes[at] = code[row, head][:, 0::2] | code[row, head][:, 1::2] << 4
            scales = getattr(cache, name + "_scale").copy()
            scales[at] = scale[row, head]
            assert np.array_equal(cache.dev[name + "_scale"].cpu().numpy(), scales)
            got = cache.dev[name].cpu().numpy()
            assert np.array_equal(got, codes)
            want = np.zeros((n, hkv, hd))
            want[row, head] = R.decode(code, scale)[row, head]
            assert np.array_equal(out.double().cpu().numpy().reshape(n, hkv, hd), want, equal_nan=True)
        weight, position = cache.weight.copy(), cache.position.copy()
        weight[at], position[at] = 0.0, positions[row]
        assert np.array_equal(cache.dev["weight"].cpu().numpy(), weight, equal_nan=True)
        assert np.array_equal(cache.dev["position"].cpu().numpy(), position)


def test_no_value_is_off_by_more_than_half_its_step(torch_mod):
    torch = torch_mod
    n, hkv, hd = 256, 2, 128
    x = (torch.randn((n, hkv * hd), generator=torch.Generator().manual_seed(3)) * 5).cuda()
    with Model(hkv, hd, False) as (B, h):
        cache = R.Cache(B, 20, hkv, 16, hd, 0, book=False)
        s = cache.upload(B)
        slots = torch.arange(n, dtype=torch.int32, device="cuda")
        ko, vo = torch.empty_like(x), torch.empty_like(x)
        B.mace_kv4_append(h, s, x, -x, slots)
        B.mace_kv4_gather(h, s, slots, ko, vo)
        torch.cuda.synchronize()
    assert torch.equal(vo, -ko)
    scale = torch.from_numpy(2.0 ** (cache.dev["k_scale"].cpu().numpy().astype(np.float64) - 127)).permute(0, 2, 1, 3).reshape(-1, hkv * hd // 32)[:n]
    y, d = ko.double().cpu().abs() / scale.repeat_interleave(32, 1), (ko - x).double().cpu().abs() / scale.repeat_interleave(32, 1)
    step = torch.where(y >= 4, 2.0, torch.where(y >= 2, 1.0, 0.5))
    assert (d <= step / 2).all()


def test_slots_of_the_last_block_of_a_large_pool(torch_mod):
    """Byte offsets beyond 2^32: the last blocks of a pool of 2^27 rows of heads."""
    torch = torch_mod
    hkv, hd, size, blocks = 8, 128, 16, 1 << 20
    with Model(hkv, hd, True) as (B, h):
        pool = lambda b: torch.zeros((blocks, hkv, size, b), dtype=torch.uint8, device="cuda")
        k, v, ks, vs = pool(64), pool(64), pool(4), pool(4)
        s = B.kv4_cache_struct(k, v, ks, vs)
        x = torch.randn((40, hkv * hd), generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
        slots = torch.arange(blocks * size - 40, blocks * size, dtype=torch.int32, device="cuda")
        ko, vo = torch.empty_like(x), torch.empty_like(x)
        B.mace_kv4_append(h, s, x, x, slots)
        B.mace_kv4_gather(h, s, slots, ko, vo)
        torch.cuda.synchronize()
        want = R.decode(*R.encode(x.double().cpu().numpy()))
        assert np.array_equal(ko.double().cpu().numpy(), want) and torch.equal(ko, vo)
        assert (k[:-3] == 0).all() and (k[-1] != 0).any()
