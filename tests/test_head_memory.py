"""What a head's forward call needs of memory, with no GPU: bounded whatever the rows and the vocabulary."""
import pytest

from paper_2410_11415_amd import binding

P = 4096


def workspace(rows, width, vocab, dtype=1, k=1, back=False):
    args = binding.klay_head_args(dtype, 0, width, vocab, k, 0, rows, P, binding.klay_rows(rows, 0, width), P, width, None, P, binding.klay_rows(rows, 0, k), 1)
    return binding.klay_head_workspace_bytes(args, back)


@pytest.mark.parametrize("rows", [1, 32, 256, 257, 600, 4096, 16384, 16385, 1 << 20])
@pytest.mark.parametrize("vocab", [10, 32771, 131072, 1 << 20, (1 << 22) - 5, 1 << 25, (1 << 31) - 4097])
def test_sums_of_tiles(rows, vocab):
    """64 MB of them, or those of one tile of rows: 16 bytes for each of at most 256 rows and every 256 tokens (128 rows: every 128)"""
    kept = binding.klay_list_kept_bytes(rows, 1)
    assert workspace(rows, 64, vocab) <= kept + max(1 << 26, 16 * min(rows, 256) * (vocab // 256 + 1), 16 * min(rows, 128) * (vocab // 128 + 1)) + 1024
