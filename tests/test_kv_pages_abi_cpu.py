"""Refusals of the calls on pages that need no GPU: every argument is checked before the device is
asked for anything, with a message."""
import ctypes

import pytest

from paper_2609_36608_amd import binding as bd
from test_paged_abi_cpu import P16, handle


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


def fork_args(**kw):
    return dict(handle=handle(), block_tables=P16, max_pages=4, seq_lens=P16, num_seqs=2, parents=P16, page_refs=P16,
                num_pages=8, stream=None) | kw


def resize_args(**kw):
    return dict(handle=handle(), block_tables=P16, max_pages=4, seq_lens=P16, new_lens=P16, num_seqs=2, page_refs=P16,
                num_pages=8, granted=P16, copies=P16, workspace=P16, workspace_bytes=48, stream=None) | kw


def copy_args(**kw):
    return dict(handle=handle(), k_pages=P16, v_pages=P16, num_pages=8, copies=P16, num_copies=3, stream=None) | kw


def compact_args(**kw):
    return dict(handle=handle(), k_pages=P16, v_pages=P16, num_pages=8, block_tables=P16, max_pages=4, seq_lens=P16,
                q_starts=P16, q_lens=P16, keep=P16, keep_lens=P16, num_seqs=2, total_q=9, new_lens=None, stream=None) | kw


CALLS = {"fork": ("ctx_kv_fork_run_paged", fork_args), "resize": ("ctx_kv_resize_run_paged", resize_args),
         "copy": ("ctx_kv_copy_run_paged", copy_args), "compact": ("ctx_kv_compact_run_paged", compact_args)}
INVALID, UNSUPPORTED, CAPACITY, ALIGNMENT = (bd.CTX_ERR_INVALID_ARG, bd.CTX_ERR_UNSUPPORTED, bd.CTX_ERR_CAPACITY,
                                             bd.CTX_ERR_ALIGNMENT)
TABLES = [(dict(num_seqs=-1), INVALID), (dict(num_seqs=5), CAPACITY), (dict(max_pages=0), INVALID),
          (dict(block_tables=None), INVALID), (dict(seq_lens=None), INVALID)]
EVERY = [(dict(handle=None), INVALID), (dict(handle=handle(page_tokens=0)), UNSUPPORTED), (dict(num_pages=-1), INVALID),
         (dict(num_pages=2 ** 27), UNSUPPORTED)]
CASES = [(call, *case) for call in CALLS for case in EVERY + (TABLES if call != "copy" else [])] + [
    ("fork", dict(parents=None), INVALID),
    ("fork", dict(page_refs=None), INVALID),
    ("resize", dict(new_lens=None), INVALID),
    ("resize", dict(page_refs=None), INVALID),
    ("resize", dict(granted=None), INVALID),
    ("resize", dict(copies=None), INVALID),
    ("resize", dict(copies=20), ALIGNMENT),
    ("resize", dict(workspace=None), INVALID),
    ("resize", dict(workspace=24), ALIGNMENT),
    ("resize", dict(workspace_bytes=47), CAPACITY),
    ("copy", dict(num_copies=-1), INVALID),
    ("copy", dict(copies=None), INVALID),
    ("copy", dict(copies=20), ALIGNMENT),
    ("copy", dict(k_pages=None), INVALID),
    ("copy", dict(v_pages=24), ALIGNMENT),
    ("compact", dict(k_pages=24), ALIGNMENT),
    ("compact", dict(v_pages=None), INVALID),
    ("compact", dict(q_starts=None), INVALID),
    ("compact", dict(q_lens=None), INVALID),
    ("compact", dict(keep=None), INVALID),
    ("compact", dict(keep_lens=None), INVALID),
    ("compact", dict(total_q=-1), INVALID),
    ("compact", dict(seq_lens=32, new_lens=32), INVALID),
    ("compact", dict(keep_lens=32, new_lens=32), INVALID),
]


@pytest.mark.parametrize("call,kw,status", CASES)
def test_refuses(lib, call, kw, status):
    name, args = CALLS[call]
    assert getattr(lib, name)(*args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


def test_nothing_to_do(lib):
    assert lib.ctx_kv_fork_run_paged(*fork_args(num_seqs=0, parents=None).values()) == bd.CTX_OK
    assert lib.ctx_kv_resize_run_paged(*resize_args(num_seqs=0, workspace=None).values()) == bd.CTX_OK
    assert lib.ctx_kv_copy_run_paged(*copy_args(num_copies=0, copies=None).values()) == bd.CTX_OK
    assert lib.ctx_kv_compact_run_paged(*compact_args(num_seqs=0, keep=None).values()) == bd.CTX_OK


def test_workspace(lib):
    assert lib.ctx_kv_resize_workspace(2, 8) == 48
    assert lib.ctx_kv_resize_workspace(0, 0) == 0 and lib.ctx_kv_resize_workspace(-3, -8) == 0
