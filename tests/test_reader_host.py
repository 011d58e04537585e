"""Host side of the reader operators: the distance buckets and the argument checks, without a GPU."""
import ctypes as C

import pytest

from paper_1606_08495_b200 import binding


def starts_in_whole_numbers(n, reach):
    """Bucket e + k starts at the least m with m^N >= e^(N-k) reach^k, e = n/2, N = n - e."""
    e = n // 2
    out = list(range(e))
    for k in range(n - e):
        m = e
        while m ** (n - e) < e ** (n - e - k) * reach ** k:
            m += 1
        out.append(m)
    return out


@pytest.mark.parametrize("n", [2, 3, 4, 5, 8, 16, 31, 32, 64])
@pytest.mark.parametrize("reach", [2, 3, 4, 16, 33, 64, 100, 128, 200, 256, 512, 1000, 1024])
def test_bucket_starts(n, reach):
    if reach <= n // 2:
        with pytest.raises(binding.W2VError):
            binding.w2v_bucket_starts(n, reach, False)
        return
    assert binding.w2v_bucket_starts(n, reach, False).tolist() == starts_in_whole_numbers(n, reach)
    if 2 * n <= 64 and n >= 2:
        assert binding.w2v_bucket_starts(2 * n, reach, True).tolist() == starts_in_whole_numbers(n, reach)


@pytest.mark.parametrize("buckets,reach,two", [(0, 128, False), (1, 128, False), (65, 128, False), (2, 128, True), (7, 128, True), (32, 16, False), (32, 1025, False)])
def test_bucket_starts_refusals(buckets, reach, two):
    with pytest.raises(binding.W2VError):
        binding.w2v_bucket_starts(buckets, reach, two)


def test_calls_without_a_handle_are_refused():
    lib = binding.load()
    w = binding.Window()
    assert lib.w2v_layer_norm(None, 0, 4, None, 4, 0, None, None, 1e-5, None, 4, 0, None, None) == binding.W2V_ERR_ARG
    assert lib.w2v_sentence_spans(None, None, 0, None) == binding.W2V_ERR_ARG
    assert lib.w2v_attend(None, C.byref(w), 0, None, None, 0, None, 0, None, 0, None, None, 0, None) == binding.W2V_ERR_ARG
    assert lib.w2v_attend_token(None, C.byref(w), 0, None, None, None, None, None, None, 0, None, None) == binding.W2V_ERR_ARG
    assert lib.w2v_fourbit_scores(None, None, 0, 0, None, None, 0, 4, 32, None, 0) == binding.W2V_ERR_ARG
    assert C.sizeof(binding.Window) == 44
