"""What the tests share: a test that compares the device's free memory has run once before it counts."""
import pytest

import test_zz_no_alloc as no_alloc
from conftest import run_once_before


def test_functions_that_compare_free_memory_run_once_before():
    runs = []

    class Device:
        @staticmethod
        def mem_get_info():
            return 1, 2

    def compares(**params):
        runs.append((params, Device.mem_get_info()))
        assert not runs, "the first run's verdict does not count"

    def other(**params):
        runs.append(params)

    run_once_before(compares, dict(n=3))
    run_once_before(other, {})
    assert runs == [(dict(n=3), (1, 2))]

    def broken():
        Device.mem_get_info()
        raise ValueError

    with pytest.raises(ValueError):
        run_once_before(broken, {})


def test_the_comparison_of_free_memory_is_such_a_function():
    f = no_alloc.test_static_scratch_matches_workspace_scratch_twice_in_a_row
    assert "mem_get_info" in f.__code__.co_names
    assert "mem_get_info" not in no_alloc.test_static_calls_of_different_sizes_share_the_array.__code__.co_names
