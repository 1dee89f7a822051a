"""What the operators on the 4-bit cache launch and how much workspace they take, by the bounds of a call, on a machine without a GPU."""
import pytest

from test_kv4_host import OK, recorder  # noqa: F401  (the fixture)


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
