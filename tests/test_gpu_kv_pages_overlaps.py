"""Calls on pages whose arrays share memory."""
import pytest
import torch

from paper_2609_36608_amd import CtxError, DecodeAttention
from test_gpu_kv_pages import caches, i32

pytestmark = pytest.mark.gpu


def test_lengths_of_one_buffer():
    """Slices of one tensor that overlap are refused, others taken."""
    state = torch.zeros(8, dtype=torch.int32).cuda()
    table, refs = torch.full((4, 2), -1, dtype=torch.int32).cuda(), torch.zeros(9, dtype=torch.int32).cuda()
    k, v = caches(1, 9, 16, 2)
    with DecodeAttention(2, 2, 4, 32, page_tokens=16) as attn:
        with pytest.raises(CtxError, match="overlap"):
            attn.resize_pages(table, state[:4], state[4:], refs, granted=state[1:5])
        with pytest.raises(CtxError, match="overlap"):
            attn.fork_pages(table, state[:4], refs, state[:4])
        with pytest.raises(CtxError, match="overlap"):
            attn.compact_paged(k, v, table, state[:4], state[4:], state[4:], state[4:], state[4:], new_lens=state[4:])
        state[4:] = 5
        granted, copies = attn.resize_pages(table, state[:4], state[4:], refs, granted=state[:4])
        assert state.tolist() == [5] * 8 and table[:, 0].tolist() == [0, 1, 2, 3] and refs.tolist() == [1] * 4 + [0] * 5
