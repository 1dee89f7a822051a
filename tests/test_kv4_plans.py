"""What the operators on the 4-bit cache launch and how much workspace they take, by the bounds of a call, on a machine without a GPU."""
import pytest

from test_kv4_host import INVALID, OK, recorder  # noqa: F401  (the fixture)


def attention(recorder, **opts):
    status, error, launches, need = recorder("attention", **{**dict(hkv=8, group=4, hd=128, blocks=1 << 16), **opts})
    assert status == OK, error
    return launches, need


@pytest.mark.parametrize("n_req,bound,splits", [(256, 16384, 1), (128, 4096, 1), (64, 4096, 1), (64, 16384, 4), (1, 131072, 64), (16, 1024, 1)])
@pytest.mark.parametrize("max_rows", [1, 2, 4])
def test_bounds_that_are_powers_of_two_have_no_split_for_their_tail(recorder, n_req, bound, splits, max_rows):
    """The rows' own tokens lie behind max_context: they belong to the last split, up to a turn of 64 of them, where there is but one or the chip is full."""
    rest = dict(n_req=n_req, max_rows=max_rows, tables=1 << 14)
    at, at_need = attention(recorder, max_context=bound, **rest)
    below, below_need = attention(recorder, max_context=bound - max_rows, **rest)
    assert [l["grid"] for l in at] == [l["grid"] for l in below] and at_need == below_need
    assert at[0]["grid"][1] == splits and len(at) == (1 if splits == 1 else 2)


def test_a_tail_in_an_idle_chip_is_a_split_of_its_own(recorder):
    launches, _ = attention(recorder, n_req=4, max_context=2048)
    assert launches[0]["grid"][1] == 3


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("hkv,group,hd", [(8, 8, 128), (1, 1, 128), (32, 1, 64), (4, 4, 128), (64, 2, 64)])
def test_states_of_splits_stay_within_a_million_rows(recorder, hkv, group, hd, bf16):
    """2^20 states of HD sums, a maximum and a sum, and a log sum a row, each part rounded up to 256 bytes; only bounds that the call takes (else the size is 0)."""
    most = 0
    for n_req in (1, 7, 64, 1024, 8192, 65535):
        for max_rows in (1, 2, 17, 300, 65535):
            for max_context in (0, 1000, 16384, 131070, 1 << 20, 1 << 26):
                need = recorder("attention", hkv=hkv, group=group, hd=hd, bf16=bf16, blocks=1000, n_req=n_req, max_rows=max_rows, max_context=max_context, tables=1)[3]
                rows = n_req * max_rows * hkv * group
                assert need <= (1 << 20) * (4 * hd + 8) + 12 * rows + 1024, (n_req, max_rows, max_context)
                most = max(most, need)
    assert most > 0


def test_the_largest_states(recorder):
    assert recorder("attention", hkv=8, group=8, hd=128, n_req=1024, max_rows=2, max_context=131070)[3] == (1 << 20) * 520 + (1 << 17) * 4


@pytest.mark.parametrize("scale,status", [(2.0**126, OK), (-(2.0**126), OK), (2.0**126 * (1 + 2.0**-23), INVALID), (3e38, INVALID), (-3e38, INVALID), ("-inf", INVALID)])
def test_scales_whose_exponents_of_two_overflow_are_refused(recorder, scale, status):
    assert recorder("attention", scale=scale)[0] == status


@pytest.mark.parametrize("magnitude,status", [(3.4028234e38, OK), (3.5e38, INVALID), (-1e300, INVALID), ("nan", INVALID)])
def test_rotary_magnitudes_that_are_infinite_in_fp32_are_refused(recorder, magnitude, status):
    assert recorder("rotary", magnitude=magnitude)[0] == status
