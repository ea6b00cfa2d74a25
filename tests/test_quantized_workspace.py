"""The 8-bit attention's workspace of prompts goes by what they can see, not by the pool."""
import pytest

from paper_2511_09844_gb300 import build, sd2


@pytest.fixture(scope="module")
def size():
    build.build()
    return sd2.load_library().sd2_attention_quantized_workspace_bytes


PAGE = 2 * 8 * 16 * 128 * 2            # a page as bf16, 8 heads of 128


@pytest.mark.parametrize("M,n_seq,max_kv,window,seen", [
    (2048, 1, 2048, 0, 128), (2048, 1, 2040, 0, 128), (2000, 4, 3000, 0, 4 * 188), (512, 1, 16000, 0, 1000),
    (4096, 8, 60000, 1024, 8 * (4096 + 1024) // 16 + 8 * 3)])
def test_prompts_need_room_for_what_they_see(size, M, n_seq, max_kv, window, seen):
    needs = [size(M, n_seq, 32, 8, 128, max_kv, n, window, 0) for n in (10000, 60000, 200000, 1000000)]
    assert len(set(needs)) == 1 or window
    # pages, a table of them, and what prompt attention asks for
    most = (seen * PAGE + n_seq * (max_kv // 16 + 1) * 4 + (64 << 10)) + sd2.load_library().sd2_attention_window_workspace_bytes(
        M, n_seq, 32, 8, 128, max_kv, window or 1 << 30, 0)
    assert max(needs) <= most
    # no more than the pool, where that is small
    assert size(M, n_seq, 32, 8, 128, max_kv, 100, window, 0) <= 100 * PAGE + most - seen * PAGE


def test_what_a_large_pool_costs(size):
    """Of a pool beyond 4 GB, at most 128 MB are widened."""
    assert size(2000, 16, 32, 8, 128, 1900, 70000, 0, 0) > 16 * 119 * PAGE
    assert size(2000, 16, 32, 8, 128, 2500, 70000, 0, 0) < 64 << 20
    assert size(2000, 16, 32, 8, 128, 2500, 60000, 0, 0) > 16 * 157 * PAGE
