"""The committed profiles that bench.py quotes belong to the committed kernels: each names the sources it was taken from
and their hash, and gives the counters that the bench line asks for."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def bench():
    spec = importlib.util.spec_from_file_location("bench_for_profiles", os.path.join(ROOT, "bench.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("profile,kernel", [
    ("replay_and_route_kernels_qwen3_30b_T16384.txt", "gemm1_wide"),
    ("replay_and_route_kernels_qwen3_30b_T16384.txt", "combine_bf16_kernel"),
    ("replay_and_route_kernels_qwen3_235b_T32768.txt", "gemm1_wide"),
    ("replay_backward_kernels_qwen3_30b_bwd_T16384.txt", "bwd_wgrad<3>"),
    ("predictor_rollout_diagnostics_kernels_qwen3_30b_T16384.txt", "router_mfma_kernel<2, 1, 0>"),
])
def test_a_profile_is_of_these_sources(bench, profile, kernel):
    assert bench.profiled_traffic(profile, kernel)
    assert "mfma_busy" in bench.profiled_counters(profile, kernel)
