"""A launch counts the threads of a dimension in 32 bits: calls that would need more workgroups are refused
before the device is asked for anything."""
import ctypes

import pytest

from paper_2609_36608_amd import binding as bd
from test_kv_pages_abi_cpu import compact_args, copy_args, fork_args, resize_args
from test_logprob_abi_cpu import BF16, grad_args, run_args
from test_paged_abi_cpu import handle
from test_tree_abi_cpu import args as tree_args

MOST = 2 ** 24 - 1  # workgroups of 256 threads


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


def refused(lib, status, what, rc):
    assert rc == status, rc
    assert what in lib.ctx_decode_attn_last_error().decode()


def test_token_logprobs(lib):
    kw = dict(num_rows=MOST + 1, logits=4096, stream=None)
    refused(lib, bd.CTX_ERR_UNSUPPORTED, "num_rows", lib.ctx_token_logprob_run(*run_args(**kw).values()))
    refused(lib, bd.CTX_ERR_UNSUPPORTED, "num_rows",
            lib.ctx_token_logprob_grad_run(*grad_args(**kw, grad_logits=2 ** 40).values()))
    size = ctypes.c_size_t()
    refused(lib, bd.CTX_ERR_UNSUPPORTED, "num_rows",
            lib.ctx_token_logprob_workspace(BF16, 100, MOST + 1, 0, ctypes.byref(size)))


def test_pages(lib):
    many = handle(max_batch=2 ** 26)
    for name, args in (("ctx_kv_fork_run_paged", fork_args), ("ctx_kv_resize_run_paged", resize_args)):
        refused(lib, bd.CTX_ERR_INVALID_ARG, "grid", getattr(lib, name)(*args(handle=many, num_seqs=MOST + 1).values()))
    # pages of 32 KiB in one workgroup each, 48 KiB in two
    refused(lib, bd.CTX_ERR_INVALID_ARG, "grid", lib.ctx_kv_copy_run_paged(*copy_args(num_copies=MOST + 1).values()))
    refused(lib, bd.CTX_ERR_INVALID_ARG, "grid",
            lib.ctx_kv_copy_run_paged(*copy_args(handle=handle(page_tokens=48), num_copies=MOST // 2 + 1).values()))
    refused(lib, bd.CTX_ERR_INVALID_ARG, "grid",
            lib.ctx_kv_compact_run_paged(*compact_args(handle=many, num_seqs=MOST // 16 + 1).values()))


def test_trees(lib):
    # 16 drafts of 2 heads each are 2 workgroups of the join, for each of 8 KV heads
    kw = dict(handle=handle(max_batch=2 ** 26), max_q_len=16, num_seqs=MOST // 16 + 1)
    refused(lib, bd.CTX_ERR_INVALID_ARG, "grid", lib.ctx_tree_attn_run_paged(*tree_args(**kw).values()))
    size = ctypes.c_size_t()
    refused(lib, bd.CTX_ERR_INVALID_ARG, "grid",
            lib.ctx_tree_attn_workspace(kw["handle"], kw["num_seqs"], 16, ctypes.byref(size)))
