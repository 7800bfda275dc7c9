"""What the step of a 4-bit row's group, a product by the nearest fp32 of 1/15 rounded up, means for values that lie on a grid of
16 levels already: the numbers the header gives."""
import pytest
import torch

import pack4_reference as ref


def grid(step):
    x = torch.zeros(64)
    x[:16] = torch.arange(16) * step
    return x


def test_grids_of_every_significand():
    steps = torch.arange(128).mul(2.0 ** -7).add(1.0).bfloat16().float()
    larger = 0
    for s in steps:
        c, got, b = ref.pack(grid(s))
        assert float(got[0, 0]) in (float(s), float(torch.nextafter(s.bfloat16(), torch.tensor(4.0).bfloat16())))
        larger += float(got[0, 0]) != float(s)
        values = ref.values(grid(s))
        assert ((values - grid(s)).abs() <= ref.error_bound(grid(s))).all()
        if float(got[0, 0]) == float(s):
            assert torch.equal(values, grid(s))
    assert larger == 109


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_stored_again_values_are_off_by_as_much_once_more(dtype):
    x = torch.randn(500, 128, generator=torch.Generator().manual_seed(0)).to(dtype)
    once = ref.values(x)
    again = ref.values(once)
    assert not torch.equal(once, again)
    assert ((again.double() - once.double()).abs() <= ref.error_bound(once)).all()


def test_header_says_so():
    from test_sources_cpu import header_before

    words = header_before("kvs_status kvs_set_cache_format(")
    assert "109 of the 128" in words and "stored in one again" in words
