"""CPU-only, under the address and undefined-behaviour sanitizers: how attention of few new tokens over the cache shares out its work."""
from test_sanitizers import _host_build_of_kernel_headers


def test_shares_are_as_defined_and_stay_in_range_whatever_the_arrays_hold(tmp_path):
    res = _host_build_of_kernel_headers(tmp_path, "attn_shares")
    assert res.returncode == 0 and "in range" in res.stdout, res.stdout
