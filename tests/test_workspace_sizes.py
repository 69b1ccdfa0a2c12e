"""What the fused cross entropy asks of its caller (host side: no GPU)."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2509_06980_b200 import build
    build.build()
    from paper_2509_06980_b200 import binding
    return binding


def _scratch(T, V):
    return 2 * min((T + 255) // 256 * 256, 18944) * ((V + 255) // 256 * 256)


def _rows(T, D):
    """The copies of the hidden states (two), bf16."""
    return 2 * 2 * ((T + 255) // 256 * 256) * D


@pytest.mark.parametrize("T,D,V", [(8192, 4096, 512), (2047, 2048, 512), (40000, 64, 264), (1, 64, 8), (300, 8192, 7936)])
def test_no_partial_sums_where_the_vocabulary_is_not_cut(b, T, D, V):
    """A piece of grad_hidden's sum covers at least 1024 columns; with fewer than 2048 there is one piece, and what is kept
    beside the scratch and the rows is small: the tokens' records, the sweep's partials (80 per token), column sums."""
    n = b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY, T, V, D, b.RLF_F32)
    pieces = 0 if V < 2048 else 4 * (V // 1024) * min(T + 255, 18944) * D
    assert n <= _scratch(T, V) + _rows(T, D) + pieces + T * (8 * 80 + 128) + 4 * D * 140 + 4 * T * (V // 256 + 2) + (1 << 16)


@pytest.mark.parametrize("T,D,V", [(64, 2560, 151936), (2047, 2048, 32000), (8192, 4096, 151936), (1, 8192, 262144), (512, 4096, 50304)])
def test_partial_sums_stay_below_the_scratch(b, T, D, V):
    n = b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY, T, V, D, b.RLF_F32)
    beside = n - _scratch(T, V) - _rows(T, D) - T * (8 * 80 + 128) - 4 * D * 140 - 4 * T * (V // 256 + 2)
    assert beside <= _scratch(T, V)


@pytest.mark.parametrize("T,D,V", [(8192, 4096, 151936), (64, 2560, 151936), (40000, 64, 264), (0, 64, 8)])
def test_a_call_without_gradients_keeps_no_scratch(b, T, D, V):
    n = b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY_FWD, T, V, D, b.RLF_F32)
    assert 0 < n <= _rows(T, D) // 2 + T * (8 * 80 + 128) + 4 * D * 140 + (1 << 16)
    assert n == b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY_FWD, T, V, D, b.RLF_BF16)
    assert n < b.workspace_bytes(b.FN_FUSED_CROSS_ENTROPY, T, V, D, b.RLF_F32)
