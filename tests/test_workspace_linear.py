"""What the backward of the linear layer asks of its caller, against what its kernels write there (host side: no GPU).

A W of 1 to 4 rows may be that of a plain layer with as many outputs, whose weight gradient is summed from partial rows in fp32,
or, an even number, of a gated layer with half as many, which keeps gz, the gradient before the activation, in bf16 like any other."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2509_06980_b200 import build
    build.build()
    from paper_2509_06980_b200 import binding
    return binding


@pytest.mark.parametrize("T,D", [(1, 8), (7, 64), (33, 2560), (300, 8), (4096, 8), (5000, 64), (32768, 64), (32768, 4096), (1 << 20, 8), (1 << 29, 64)])
@pytest.mark.parametrize("rows", list(range(1, 17)) + [260, 2560])
def test_everything_has_room_of_its_own(b, T, D, rows):
    n = b.workspace_bytes(b.FN_LINEAR_BWD, T, rows, D, b.RLF_BF16)
    gz = 2 * T * ((rows + 7) // 8 * 8)                          # bf16, rows of whole 16-byte vectors
    bias = 4 * rows * min(256, (T + 31) // 32)                  # a partial row per slice of tokens
    if rows in (1, 3):                                          # (no gated layer's)
        gz = 0
    assert n >= gz + bias and n % 256 == 0
    if rows <= 4:
        assert n >= 4 * rows * (D + 1) * min(256, (T + 7) // 8)


def test_few_rows_keep_nothing_large(b):
    """Beside the partial rows a W of two or four rows keeps 16 bytes a token, one of one or three nothing."""
    for T, D, rows in ((8191, 4096, 1), (32768, 2560, 2), (32768, 64, 4), (0, 64, 2)):
        assert b.workspace_bytes(b.FN_LINEAR_BWD, T, rows, D, b.RLF_BF16) <= (0 if rows % 2 else 16 * T) + 4 * rows * (D + 1) * 256 + 1024
