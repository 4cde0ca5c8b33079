"""The packed arena's entry points (include/kvr_packed.h) at sizes that only large calls
reach: steps that the decode over it does not take."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_14635_amd import kvr  # noqa: E402
from paper_2608_14635_amd import workloads as W  # noqa: E402

import packed_util as P  # noqa: E402


def bound(shape, B, blocks):
    n = kvr.kv_packed_bytes(shape, B, blocks)
    raw = torch.empty(n, dtype=torch.uint8, device="cuda")
    return raw, kvr.kv_packed_bind(raw.data_ptr(), n, shape, B, blocks)


def step_status(shape, handle, positions, tables, size):
    """What a step with a workspace of `size` bytes that is never touched answers."""
    w = kvr.Weights(kvr.make_desc(shape), 0x1000, [{k: 0x1000 for k in kvr.LAYER_FIELDS}] * shape.num_layers)
    with pytest.raises(kvr.KvError) as e:
        kvr.kv_packed_decode_step(w, 0x1000, 0x1000, np.zeros(len(positions), np.int32), positions, tables, handle,
                                  0x10000, size, 0x2000)
    assert e.value.message
    return e.value.status


@pytest.mark.gpu
def test_decode_steps_of_positions_that_the_attention_does_not_take():
    """Requests whose tables name one block over and over, but for the block that they write."""
    shape, B = dataclasses.replace(W.TINY_BF16, num_layers=1), 1 << 14
    raw, h = bound(shape, B, 41)
    top = (1 << 31) - 1

    def tables(n):
        t = np.zeros((n, (1 << 31) // B), np.int32)
        t[:, -1] = np.arange(1, n + 1)
        return t
    assert step_status(shape, h, [top], tables(1), 1 << 62) == kvr.KV_EINVAL
    assert step_status(shape, h, [5, top], np.vstack([np.full(1 << 17, 7, np.int32), tables(1)[0]]), 1 << 62) == kvr.KV_EINVAL
    assert step_status(shape, h, [top - 1] * 40, tables(40), 1 << 62) == kvr.KV_EINVAL
    # one position less, and fewer requests: the workspace is what is missing
    assert step_status(shape, h, [top - 1], tables(1), 16) == kvr.KV_ENOMEM
    assert step_status(shape, h, [top - 1] * 8, tables(8), 16) == kvr.KV_ENOMEM
    kvr.kv_packed_release(h)


@pytest.mark.gpu
def test_decode_steps_of_more_requests_than_the_attention_takes():
    shape, n = dataclasses.replace(P.F32[32], num_layers=1, num_q_heads=4, num_kv_heads=4), (1 << 24) + 1
    raw, h = bound(shape, 16, n)
    assert step_status(shape, h, np.zeros(n, np.int32), np.arange(n, dtype=np.int32)[:, None], 1 << 62) == kvr.KV_EINVAL
    kvr.kv_packed_release(h)
