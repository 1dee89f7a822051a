"""Attention over the 4-bit paged cache and eviction from it at the borders of what their documentation says: errors, NaN, infinities, missing blocks."""
import numpy as np
import pytest

import kv4_reference as R
from test_gpu_kv4_attention import workspace
from test_gpu_kv4_cache import Model

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
