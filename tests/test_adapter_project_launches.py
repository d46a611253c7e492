"""Launches of the projection with adapters that would have 2^32 threads are refused with the sizes (no GPU)."""

import pytest

from paper_2607_20940_amd import mssa


def _size(rows, parts, rank, segments=1):
    return mssa.mssa_adapter_project_workspace_size(
        mssa.adapter_project_desc(rows, 8, 8, segments, 1, rank, parts=parts))


# Tiles of 64 rows, 256 threads for each 96 of the parts' rank columns: 2^24 / columns tiles are 2^32 threads.
@pytest.mark.parametrize("rows,parts,rank", [(1 << 26, 8, 256), (1 << 26, 8, 192), (64 * ((1 << 24) // 22 + 1), 8, 256)])
def test_too_many_blocks_of_low_rank_factors_are_refused(rows, parts, rank):
    with pytest.raises(mssa.MssaError) as e:
        _size(rows, parts, rank)
    assert e.value.status == mssa.MSSA_ERR_UNSUPPORTED, str(e.value)


@pytest.mark.parametrize("rows,parts,rank", [(64 * ((1 << 24) // 22 - 1), 8, 256), (1 << 26, 1, 256), (1 << 26, 2, 16)])
def test_the_most_blocks_of_low_rank_factors(rows, parts, rank):
    assert _size(rows, parts, rank) >= rows * parts * rank * 2
