"""The host-only checks (kv_rebuild_check, kv_rebuild_from_check, kv_decode_check) of
arenas with more blocks than host memory holds numbers: what they need goes by the
blocks that are written."""
import pytest

from paper_2608_14635_amd import kvr
from paper_2608_14635_amd import workloads as W

MANY = [1 << 40, 1 << 60, (1 << 63) - 1]
S = W.TINY_BF16


@pytest.mark.parametrize("blocks", MANY)
def test_decode_check(blocks):
    check = lambda pos, tab: kvr.kv_decode_check(S, 16, blocks, [1] * len(pos), pos, tab)  # noqa: E731
    assert check([0], [[0]]) == kvr.KV_OK
    assert check([40, 3], [[5, 1 << 20, 7], [9, -1, -1]]) == kvr.KV_OK
    assert check([40, 3], [[5, 6, 7], [7, -1, -1]]) == kvr.KV_EALIAS
    assert check([40, 3], [[5, 9, 7], [9, -1, -1]]) == kvr.KV_EALIAS
    assert check([40, 3], [[1 << 30, 1 << 30, 7], [9, -1, -1]]) == kvr.KV_OK
    assert check([40], [[5, -1, 7]]) == kvr.KV_ERANGE


@pytest.mark.parametrize("blocks", MANY)
def test_rebuild_checks(blocks):
    check = lambda lens, tab: kvr.kv_rebuild_check(S, 16, blocks, [1] * sum(lens), lens, tab)  # noqa: E731
    assert check([17, 3], [[0, 1 << 20], [7, -1]]) == kvr.KV_OK
    assert check([17, 3], [[0, 7], [7, -1]]) == kvr.KV_EALIAS
    assert check([17, 3], [[0, -2], [7, -1]]) == kvr.KV_ERANGE
    # the first block of the second request is read: written by the first, in order, or by nobody
    some = lambda starts, tab: kvr.kv_rebuild_from_check(S, 16, blocks, [1] * (40 - sum(starts)), [20, 20], starts, tab)  # noqa: E731
    assert some([0, 16], [[3, 4], [3, 5]]) == kvr.KV_OK
    assert some([0, 16], [[3, 4], [1 << 30, 5]]) == kvr.KV_OK
    assert some([16, 0], [[3, 4], [3, 5]]) == kvr.KV_EALIAS
