"""Refusals of the tree attention that need no GPU: every argument is checked before the device is
asked for anything, with a message."""
import ctypes

import pytest

from paper_2609_36608_amd import binding as bd
from test_paged_abi_cpu import P16, handle, scores

INVALID, UNSUPPORTED, CAPACITY, ALIGNMENT = (bd.CTX_ERR_INVALID_ARG, bd.CTX_ERR_UNSUPPORTED, bd.CTX_ERR_CAPACITY,
                                             bd.CTX_ERR_ALIGNMENT)


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


def args(**kw):
    return dict(handle=handle(), q=P16, k_pages=P16, v_pages=P16, num_pages=8, block_tables=P16, max_pages=4, seq_lens=P16,
                q_starts=P16, q_lens=P16, parents=P16, num_seqs=2, total_q=10, max_q_len=6, scale=0.1, scores=None, out=P16,
                workspace=P16, workspace_bytes=1 << 30, stream=None) | kw


@pytest.mark.parametrize("kw,status", [
    (dict(handle=None), INVALID),
    (dict(handle=handle(page_tokens=0)), UNSUPPORTED),
    (dict(num_seqs=-1), INVALID),
    (dict(num_seqs=5), CAPACITY),
    (dict(scale=float("nan")), INVALID),
    (dict(num_pages=-1), INVALID),
    (dict(num_pages=2 ** 27), UNSUPPORTED),
    (dict(max_pages=0), INVALID),
    (dict(total_q=-1), INVALID),
    (dict(max_q_len=-1), INVALID),
    (dict(max_q_len=257), UNSUPPORTED),
    (dict(scores=scores(softcap=-1.0)), INVALID),
    (dict(scores=scores(window=-1)), INVALID),
    (dict(scores=scores(doc_starts=P16)), INVALID),
    (dict(workspace=None), INVALID),
    (dict(workspace=24), ALIGNMENT),
    (dict(workspace_bytes=100), CAPACITY),
] + [({name: None}, INVALID) for name in ("q", "k_pages", "v_pages", "block_tables", "seq_lens", "q_starts", "q_lens",
                                          "parents", "out")]
  + [({name: 24}, ALIGNMENT) for name in ("q", "k_pages", "v_pages", "out")])
def test_refuses(lib, kw, status):
    assert lib.ctx_tree_attn_run_paged(*args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


def test_nothing_to_do(lib):
    for kw in (dict(num_seqs=0), dict(max_q_len=0), dict(total_q=0)):
        assert lib.ctx_tree_attn_run_paged(*args(q=None, workspace=None, **kw).values()) == bd.CTX_OK


def test_workspace(lib):
    size = ctypes.c_size_t()
    assert lib.ctx_tree_attn_workspace(handle(), 2, 6, ctypes.byref(size)) == bd.CTX_OK and size.value > 0
    assert lib.ctx_tree_attn_workspace(handle(), 0, 6, ctypes.byref(size)) == bd.CTX_OK and size.value == 0
    for a, status in (((None, 2, 6), INVALID), ((handle(), 5, 6), CAPACITY), ((handle(), 2, 300), UNSUPPORTED),
                      ((handle(), 2, -1), INVALID), ((handle(page_tokens=0), 2, 6), UNSUPPORTED)):
        assert lib.ctx_tree_attn_workspace(*a, ctypes.byref(size)) == status
    assert lib.ctx_tree_attn_workspace(handle(), 2, 6, None) == INVALID
