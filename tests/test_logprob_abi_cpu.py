"""Refusals of the token log probability calls that need no GPU: every argument is checked before the
device is asked for anything, with a message."""
import ctypes

import pytest
import torch

from paper_2609_36608_amd import binding as bd

P16 = 16  # an aligned address; never read
BF16, F32 = bd.CTX_DTYPE_BF16, bd.CTX_DTYPE_F32


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


def run_args(**kw):
    a = dict(logits=P16, dtype=BF16, row_stride=104, vocab=100, tokens=P16, num_tokens=1, mask=None, num_rows=3, scale=1.0,
             top=2, token_logp=P16, entropy=None, stats=None, top_tokens=P16, top_logp=P16, workspace=None,
             workspace_bytes=0, stream=None)
    a.update(kw)
    return a


def grad_args(**kw):
    a = dict(logits=P16, dtype=BF16, row_stride=104, vocab=100, tokens=P16, num_tokens=1, mask=None, num_rows=3, scale=1.0,
             stats=P16, entropy=P16, grad_logp=P16, grad_entropy=P16, grad_logits=P16, grad_row_stride=104, stream=None)
    a.update(kw)
    return a


BOTH = [
    (dict(logits=None), bd.CTX_ERR_INVALID_ARG),
    (dict(dtype=2), bd.CTX_ERR_INVALID_ARG),
    (dict(vocab=0), bd.CTX_ERR_INVALID_ARG),
    (dict(vocab=-5), bd.CTX_ERR_INVALID_ARG),
    (dict(vocab=2**28 + 1, row_stride=2**29), bd.CTX_ERR_UNSUPPORTED),
    (dict(row_stride=96), bd.CTX_ERR_INVALID_ARG),
    (dict(row_stride=100), bd.CTX_ERR_INVALID_ARG),
    (dict(dtype=F32, row_stride=102), bd.CTX_ERR_INVALID_ARG),
    (dict(num_tokens=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(num_tokens=65), bd.CTX_ERR_UNSUPPORTED),
    (dict(num_tokens=0), bd.CTX_ERR_INVALID_ARG),  # with tokens
    (dict(tokens=None), bd.CTX_ERR_INVALID_ARG),
    (dict(num_rows=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(num_rows=2**24 + 1), bd.CTX_ERR_UNSUPPORTED),
    (dict(scale=0.0), bd.CTX_ERR_INVALID_ARG),
    (dict(scale=-1.0), bd.CTX_ERR_INVALID_ARG),
    (dict(scale=float("nan")), bd.CTX_ERR_INVALID_ARG),
    (dict(scale=float("inf")), bd.CTX_ERR_INVALID_ARG),
    (dict(scale=1e-31), bd.CTX_ERR_INVALID_ARG),
    (dict(logits=24), bd.CTX_ERR_ALIGNMENT),
]


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(top=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(top=65), bd.CTX_ERR_UNSUPPORTED),
    (dict(top=0), bd.CTX_ERR_INVALID_ARG),  # with outputs
    (dict(top_tokens=None), bd.CTX_ERR_INVALID_ARG),
    (dict(top_logp=None), bd.CTX_ERR_INVALID_ARG),
    (dict(token_logp=None), bd.CTX_ERR_INVALID_ARG),
    (dict(workspace=24), bd.CTX_ERR_ALIGNMENT),
])
def test_run_refuses(lib, kw, status):
    assert lib.ctx_token_logprob_run(*run_args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(grad_row_stride=96), bd.CTX_ERR_INVALID_ARG),
    (dict(grad_row_stride=108), bd.CTX_ERR_INVALID_ARG),
    (dict(stats=None), bd.CTX_ERR_INVALID_ARG),
    (dict(entropy=None), bd.CTX_ERR_INVALID_ARG),
    (dict(grad_entropy=None), bd.CTX_ERR_INVALID_ARG),
    (dict(grad_logp=None), bd.CTX_ERR_INVALID_ARG),
    (dict(grad_logits=None), bd.CTX_ERR_INVALID_ARG),
    (dict(grad_logits=40), bd.CTX_ERR_ALIGNMENT),
])
def test_grad_refuses(lib, kw, status):
    assert lib.ctx_token_logprob_grad_run(*grad_args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


@pytest.mark.parametrize("kw", [
    dict(grad_logits=4096),  # the logits themselves
    dict(grad_logits=4096 + 192),  # the last 4 columns of a row
    dict(grad_logits=4096 + 2 * 208 + 192, grad_row_stride=512),  # of the last one
    dict(grad_logits=4096 - 400),
    dict(row_stride=208, grad_row_stride=208, grad_logits=4096 + 416 + 192),  # between rows, not far enough
    dict(num_rows=1, row_stride=2**20, grad_row_stride=2**20, grad_logits=4096 + 96),
    dict(dtype=F32, grad_logits=4096 + 384),
])
def test_grad_refuses_to_overwrite_the_logits(lib, kw):
    assert lib.ctx_token_logprob_grad_run(*grad_args(logits=4096, **kw).values()) == bd.CTX_ERR_INVALID_ARG
    assert "overlaps" in lib.ctx_decode_attn_last_error().decode()


def test_no_rows(lib):
    assert lib.ctx_token_logprob_run(*run_args(num_rows=0, logits=None, tokens=None, top_tokens=None).values()) == bd.CTX_OK
    assert lib.ctx_token_logprob_grad_run(*grad_args(num_rows=0, logits=None, stats=None).values()) == bd.CTX_OK
    size = ctypes.c_size_t(7)
    assert lib.ctx_token_logprob_workspace(BF16, 100, 0, 5, ctypes.byref(size)) == bd.CTX_OK and size.value == 0


@pytest.mark.parametrize("args,status", [
    ((2, 100, 4, 0), bd.CTX_ERR_INVALID_ARG),
    ((BF16, 0, 4, 0), bd.CTX_ERR_INVALID_ARG),
    ((BF16, 100, -4, 0), bd.CTX_ERR_INVALID_ARG),
    ((BF16, 100, 4, -1), bd.CTX_ERR_INVALID_ARG),
    ((BF16, 100, 4, 65), bd.CTX_ERR_UNSUPPORTED),
])
def test_workspace_refuses(lib, args, status):
    size = ctypes.c_size_t()
    assert lib.ctx_token_logprob_workspace(*args, ctypes.byref(size)) == status
    assert lib.ctx_decode_attn_last_error().decode()
    assert lib.ctx_token_logprob_workspace(*args, None) == bd.CTX_ERR_INVALID_ARG


def test_binding_refuses_host_tensors_and_other_types():
    z = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="cuda"):
        bd.token_logprobs(z)
    with pytest.raises(TypeError):
        bd.token_logprobs(z.half())
    with pytest.raises(ValueError, match="cuda"):
        bd.token_logprobs_grad(z, None, {}, None)
