"""How much work memory the loss over a vocabulary asks for, without a GPU: a bounded room for a piece of the softmax's gradient, whatever the number of logits."""
import pytest

import paper_1802_04434_amd as ss

MIB = 1 << 20


def wanted(T, V, K):
    return ss.load_library().ss_cross_entropy_scratch_bytes(T, V, K)


def test_less_than_the_logits_would_take():
    """in 16 bits, from 2^28 of them on; half of that from 2^30 on"""
    for T, V, K in ((8192, 32768, 1024), (4096, 65536, 2048), (2048, 131072, 1024), (8192, 128000, 512), (8192, 128000, 4096), (16384, 128000, 4096), (32768, 250000, 4096)):
        logits = 2 * T * V
        assert wanted(T, V, K) < (logits if T * V < 1 << 30 else logits // 2), (T, V, K)


@pytest.mark.parametrize("T,V,K,most", [(1, 32000, 2048, 140), (1, 128000, 4096, 140), (64, 128000, 2048, 290), (1024, 128000, 4096, 350), (4096, 32000, 2048, 340), (8192, 128000, 4096, 720)])
def test_sizes(T, V, K, most):
    assert wanted(T, V, K) <= most * MIB


def test_no_more_than_its_parts():
    """D's piece and the copied weights in their room, or in that of the 1024 tokens that a piece has at the least; h; dh's sum over the pieces; the partial sums of a long product, whose
    tiles fill the card's 256 compute units once: 64 squared, 128 squared and 256 squared, four, two and one each, 2^24 entries at most; or the statistics, 8 bytes for each 32 columns of a row"""
    up = lambda n: -(-n // 64) * 64  # noqa: E731
    for T in (1, 2, 63, 64, 65, 500, 1023, 1024, 4097, 20_000, 300_000):
        for V in (1, 1000, 1024, 1025, 9999, 32_000, 128_256, 1_000_000):
            for K in (1, 64, 520, 2048, 4096, 60_001):
                if up(T) * up(K) > 1 << 34:
                    continue
                room = 2 * max(min(max(up(T) * V // 2, 1 << 27), 1 << 28), 1024 * (up(T) + up(K)), 2 * 1024 * up(K))
                room = min(room, 2 * up(V) * (up(T) + up(K)))
                statistics = 8 * T * 2 * (V // 64 + 1 + V // 1024 + 1)
                assert wanted(T, V, K) <= room + 2 * up(T) * up(K) + 4 * T * K + max(64 * MIB, statistics) + 8 * T + 16 * 256, (T, V, K)
