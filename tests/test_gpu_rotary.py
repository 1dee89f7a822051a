"""Rotary positions through the C ABI against their definition."""


import numpy as np
import pytest

pytestmark = pytest.mark.gpu


class Model:
    def __init__(self, hd, bf16):
        from paper_2510_03283_amd import binding as B
        self.B, self.h = B, B.mace_create(256, 4, 2, hd, 64, 64, 1e-6, 1e4, B.MACE_BF16 if bf16 else B.MACE_F32)

    def __enter__(self):
        return self.B, self.h

    def __exit__(self, *_):
        self.B.mace_destroy(self.h)


def reference(x, positions, freq, heads, hd, interleaved, magnitude, inverse):
    """float64 [n, heads * hd], and |a| + |b| of every element's pair (0 behind the turned part)."""
    n, rot = x.shape[0], 2 * len(freq)
    y = x[:, :heads * hd].astype(np.float64).reshape(n, heads, hd).copy()
    size = np.zeros_like(y)
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    t = positions.astype(np.float64)[:, None, None] * freq * (-1 if inverse else 1)
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = magnitude * (u * np.cos(t) - v * np.sin(t)), magnitude * (v * np.cos(t) + u * np.sin(t))
    size[..., a] = size[..., b] = abs(magnitude) * (np.abs(u) + np.abs(v))
    return y.reshape(n, -1), size.reshape(n, -1)


CASES = [  # n, heads, hd, rot, interleaved, inverse, columns of x, of out, in place
    (1, 1, 64, 64, False, False, 64, 64, False), (32, 40, 64, 64, False, False, 2816, 2560, False), (5, 3, 128, 128, True, False, 400, 384, False),
    (7, 6, 64, 2, False, True, 384, 390, False), (9, 2, 128, 24, False, False, 256, 264, False), (9, 2, 64, 24, True, True, 136, 128, False),
    (3, 5, 64, 36, False, False, 321, 323, False), (11, 4, 128, 62, True, False, 512, 515, False), (1500, 4, 64, 32, True, False, 256, 256, True),
    (4099, 2, 128, 128, False, True, 264, 264, True), (130, 64, 128, 64, False, False, 8192, 8192, True), (6, 4096, 64, 16, False, False, 262144, 262144, False),
    (2, 7, 64, 6, False, False, 449, 449, True),
]


MANY_HEADS = [  # rows of more accesses than the square root of 2^32, where a quotient by a 32-bit reciprocal is no longer exact by itself
    (3, 4095, 128, 2, True, False, 524160, 524160, False), (2, 3001, 128, 24, False, False, 384128, 384131, False), (2050, 733, 128, 2, False, False, 93824, 93825, False),
    (3, 4093, 64, 2, False, True, 261952, 261953, True),
]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("case", MANY_HEADS, ids=lambda c: "-".join(map(str, c)))
def test_rows_of_many_heads(torch_mod, bf16, case):
    test_against_the_definition(torch_mod, bf16, case)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_the_definition(torch_mod, bf16, case):
    torch = torch_mod
    n, heads, hd, rot, inter, inverse, cols, out_cols, in_place = case
    gen = torch.Generator().manual_seed(n * heads + rot)
    dtype = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn((n, cols), generator=gen).to(dtype)
    positions = torch.randint(0, 200000, (n,), generator=gen, dtype=torch.int32)
    positions[: n // 3] = torch.arange(n // 3, dtype=torch.int32)
    with Model(hd, bf16) as (B, h):
        freq = B.mace_rotary_frequencies(rot, 1e4, 4.0, 4096)
        dx = x.cuda()
        out = dx if in_place else torch.full((n, out_cols), 7.0, dtype=dtype, device="cuda")
        B.mace_rotary(h, dx, positions.cuda(), torch.from_numpy(freq).cuda(), out, heads, interleaved=inter, magnitude=1.25, inverse=inverse)
        torch.cuda.synchronize()
    want, size = reference(x.double().numpy(), positions.numpy(), freq, heads, hd, inter, 1.25, inverse)
    got = out.double().cpu().numpy()
    # (cos, sin) rounded once, two products and a sum: 4 roundings to fp32 relative to |a| + |b|, then one to the type
    tol = 4 * 2.0**-24 * size + ((2.0**-8 if bf16 else 2.0**-24) * np.abs(want) + 2.0**-140) * (size > 0)
    assert (np.abs(got[:, :heads * hd] - want) <= tol).all()
    rest = got[:, heads * hd:]
    assert (rest == (x.double().numpy()[:, heads * hd:] if in_place else 7.0)).all()            # columns behind the heads


def test_there_and_back_and_the_gradient(torch_mod):
    """inverse is the transposed map: <R x, y> = <x, R^T y>, and R^T R = magnitude^2."""
    torch = torch_mod
    n, heads, hd = 33, 5, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.randn((n, heads * hd), generator=gen, device="cuda") for _ in range(2))
    pos = torch.randint(-1000, 100000, (n,), generator=gen, device="cuda", dtype=torch.int32)
    with Model(hd, False) as (B, h):
        freq = torch.from_numpy(B.mace_rotary_frequencies(96, 5e5)).cuda()
        for inter in (False, True):
            rx, rty, back = (torch.empty_like(x) for _ in range(3))
            B.mace_rotary(h, x, pos, freq, rx, heads, interleaved=inter, magnitude=1.5)
            B.mace_rotary(h, y, pos, freq, rty, heads, interleaved=inter, magnitude=1.5, inverse=True)
            B.mace_rotary(h, rx, pos, freq, back, heads, interleaved=inter, magnitude=1.5, inverse=True)
            torch.cuda.synchronize()
            a, b = (rx.double() * y.double()).sum(), (x.double() * rty.double()).sum()
            assert abs(a - b) <= 8 * 2.0**-24 * 1.5 * x.double().norm() * y.double().norm()
            turned = back.view(n, heads, hd)[..., :96].double() - 2.25 * x.view(n, heads, hd)[..., :96].double()
            assert turned.abs().max() <= 16 * 2.0**-24 * 2.25 * 2 * x.abs().max()
            assert torch.equal(back.view(n, heads, hd)[..., 96:], x.view(n, heads, hd)[..., 96:])
            # the gradient against differences of the function itself, which is linear
            e = 2.0**-3
            moved = torch.empty_like(x)
            B.mace_rotary(h, x + e * y, pos, freq, moved, heads, interleaved=inter, magnitude=1.5)
            w = torch.randn((n, heads * hd), generator=gen, device="cuda")
            g = torch.empty_like(w)
            B.mace_rotary(h, w, pos, freq, g, heads, interleaved=inter, magnitude=1.5, inverse=True)
            torch.cuda.synchronize()
            slope = ((moved.double() - rx.double()) * w.double()).sum() / e
            assert abs(slope - (g.double() * y.double()).sum()) <= 64 * 2.0**-24 / e * 1.5 * (x.double().norm() + y.double().norm()) * w.double().norm()


def test_far_positions_keep_their_angle(torch_mod):
    torch = torch_mod
    x = torch.zeros((6, 64), device="cuda")
    x[:, :32] = 1.0
    pos = torch.tensor([0, 1, -5, 2**31 - 1, -2**31, 123456789], dtype=torch.int32, device="cuda")
    with Model(64, False) as (B, h):
        freq = B.mace_rotary_frequencies(64, 1e4)
        out = torch.empty_like(x)
        B.mace_rotary(h, x, pos, torch.from_numpy(freq).cuda(), out, 1)
        B.mace_rotary(h, x[:0], pos[:0], torch.from_numpy(freq).cuda(), out[:0], 1)                 # no rows: nothing happens
        torch.cuda.synchronize()
    t = pos.cpu().numpy().astype(np.float64)[:, None] * freq
    # the product of position and frequency is rounded to 53 bits: up to 2^-22 at 2^31
    tol = 2.0**-23 + np.abs(t) * 2.0**-53
    got = out.double().cpu().numpy()
    assert (np.abs(got[:, :32] - np.cos(t)) <= tol).all() and (np.abs(got[:, 32:] - np.sin(t)) <= tol).all()


def test_the_layers_own_embedding(torch_mod):
    """Half layout, whole head, plain frequencies: the definition that the layer uses (positions times theta^(-2i/hd))."""
    torch = torch_mod
    from oracle import mace_oracle as O
    from paper_2510_03283_amd import binding as B
    n, hd = 17, 64
    x = np.random.default_rng(0).standard_normal((n, 2, hd)).astype(np.float32)
    pos = np.arange(n) * 37
    want = O.rope(x.astype(np.float64), pos, 1e4)
    with Model(hd, False) as (_, h):
        out = torch.empty((n, 2 * hd), device="cuda")
        B.mace_rotary(h, torch.from_numpy(x.reshape(n, -1)).cuda(), torch.from_numpy(pos.astype(np.int32)).cuda(),
                      torch.from_numpy(B.mace_rotary_frequencies(hd, 1e4)).cuda(), out, 2)
        torch.cuda.synchronize()
    ref, size = reference(x.reshape(n, -1), pos, 1e4 ** (-2.0 * np.arange(hd // 2) / hd), 2, hd, False, 1.0, False)
    assert (np.abs(out.double().cpu().numpy() - ref) <= 4 * 2.0**-24 * size + 2.0**-24 * np.abs(ref)).all()
    assert np.abs(ref - want.reshape(n, -1)).max() <= 1e-12
