"""Refusals of the calls over paged caches that need no GPU: every argument is checked before the
device is asked for anything, with a message."""
import ctypes

import pytest

from paper_2609_36608_amd import binding as bd

P16 = 16  # an aligned address; never read


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


def handle(page_tokens=16, max_batch=4, hq=16, hkv=8):
    """Memory whose first member is a descriptor, as the handle's is: what the checks read."""
    mem = ctypes.create_string_buffer(256)
    desc = bd.CtxDesc(hq, hkv, 128, max_batch, 1024, bd.CTX_DTYPE_BF16, 0, page_tokens)
    ctypes.memmove(mem, ctypes.byref(desc), ctypes.sizeof(desc))
    ctypes.memset(ctypes.byref(mem, ctypes.sizeof(desc)), 0xff, 4)  # no such device
    return mem


def append_args(**kw):
    a = dict(handle=handle(), q=P16, q_stride=16 * 128, k=P16, k_stride=8 * 128, v=P16, v_stride=8 * 128, k_pages=P16,
             v_pages=P16, num_pages=8, block_tables=P16, max_pages=4, seq_lens=P16, q_starts=P16, q_lens=P16,
             num_seqs=2, total_q=10, rotary=None, q_out=P16, stream=None)
    a.update(kw)
    return a


def rotary(**kw):
    r = dict(inv_freq=P16, positions=None, q_norm=None, k_norm=None, norm_eps=1e-6, rotary_dim=128, flags=0)
    r.update(kw)
    return ctypes.byref(bd.CtxRotary(*r.values()))


@pytest.mark.parametrize("kw,status", [
    (dict(handle=None), bd.CTX_ERR_INVALID_ARG),
    (dict(handle=handle(page_tokens=0)), bd.CTX_ERR_UNSUPPORTED),
    (dict(num_seqs=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(num_seqs=5), bd.CTX_ERR_CAPACITY),
    (dict(total_q=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(num_pages=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(max_pages=0), bd.CTX_ERR_INVALID_ARG),
    (dict(q_starts=None), bd.CTX_ERR_INVALID_ARG),
    (dict(q_lens=None), bd.CTX_ERR_INVALID_ARG),
    (dict(q_starts=None, q_lens=None), bd.CTX_ERR_INVALID_ARG),  # 10 rows of 2 sequences
    (dict(q=None), bd.CTX_ERR_INVALID_ARG),
    (dict(q_out=None), bd.CTX_ERR_INVALID_ARG),
    (dict(k=None), bd.CTX_ERR_INVALID_ARG),
    (dict(v=None), bd.CTX_ERR_INVALID_ARG),
    (dict(k_pages=None), bd.CTX_ERR_INVALID_ARG),
    (dict(v_pages=None), bd.CTX_ERR_INVALID_ARG),
    (dict(block_tables=None), bd.CTX_ERR_INVALID_ARG),
    (dict(seq_lens=None), bd.CTX_ERR_INVALID_ARG),
    (dict(q_stride=15 * 128), bd.CTX_ERR_INVALID_ARG),
    (dict(k_stride=8 * 128 + 4), bd.CTX_ERR_INVALID_ARG),
    (dict(v_stride=0), bd.CTX_ERR_INVALID_ARG),
    (dict(q=32, q_out=32, q_stride=16 * 128 + 8), bd.CTX_ERR_INVALID_ARG),
    (dict(q=18), bd.CTX_ERR_ALIGNMENT),
    (dict(k=24), bd.CTX_ERR_ALIGNMENT),
    (dict(v_pages=20), bd.CTX_ERR_ALIGNMENT),
    (dict(q_out=40), bd.CTX_ERR_ALIGNMENT),
    (dict(rotary=rotary(flags=2)), bd.CTX_ERR_INVALID_ARG),
    (dict(rotary=rotary(rotary_dim=-16)), bd.CTX_ERR_INVALID_ARG),
    (dict(rotary=rotary(rotary_dim=24)), bd.CTX_ERR_UNSUPPORTED),
    (dict(rotary=rotary(rotary_dim=144)), bd.CTX_ERR_UNSUPPORTED),
    (dict(rotary=rotary(rotary_dim=0)), bd.CTX_ERR_INVALID_ARG),
    (dict(rotary=rotary(inv_freq=None)), bd.CTX_ERR_INVALID_ARG),
    (dict(rotary=rotary(q_norm=P16, norm_eps=-1.0)), bd.CTX_ERR_INVALID_ARG),
    (dict(rotary=rotary(k_norm=P16, norm_eps=float("inf"))), bd.CTX_ERR_INVALID_ARG),
    (dict(rotary=rotary(k_norm=18)), bd.CTX_ERR_ALIGNMENT),
])
def test_append_refuses(lib, kw, status):
    assert lib.ctx_kv_append_run_paged(*append_args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


def test_append_of_nothing(lib):
    assert lib.ctx_kv_append_run_paged(*append_args(num_seqs=0, total_q=0, k=None, v=None).values()) == bd.CTX_OK
    assert lib.ctx_kv_append_run_paged(*append_args(total_q=0, q=None, q_out=None).values()) == bd.CTX_OK


def prefill_args(**kw):
    a = dict(handle=handle(), q=P16, k_pages=P16, v_pages=P16, num_pages=8, block_tables=P16, max_pages=4, seq_lens=P16,
             q_starts=P16, q_lens=P16, num_seqs=2, total_q=10, max_q_len=6, scale=0.1, scores=None, out=P16, stream=None)
    a.update(kw)
    return a


def decode_args(**kw):
    a = dict(handle=handle(), q=P16, k_pages=P16, v_pages=P16, num_pages=8, block_tables=P16, max_pages=4, seq_lens=P16,
             num_seqs=2, scale=0.1, scores=None, out=P16, stream=None)
    a.update(kw)
    return a


def scores(**kw):
    s = dict(softcap=0.0, window=0, slopes=None, prefix_lens=None, doc_starts=None)
    s.update(kw)
    return ctypes.byref(bd.CtxAttnScores(*s.values()))


BOTH = [
    (dict(handle=None), bd.CTX_ERR_INVALID_ARG),
    (dict(handle=handle(page_tokens=0)), bd.CTX_ERR_UNSUPPORTED),
    (dict(num_seqs=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(num_seqs=5), bd.CTX_ERR_CAPACITY),
    (dict(scale=float("nan")), bd.CTX_ERR_INVALID_ARG),
    (dict(scale=float("inf")), bd.CTX_ERR_INVALID_ARG),
    (dict(num_pages=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(num_pages=2 ** 27), bd.CTX_ERR_UNSUPPORTED),
    (dict(max_pages=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(scores=scores(softcap=-1.0)), bd.CTX_ERR_INVALID_ARG),
    (dict(scores=scores(softcap=float("nan"))), bd.CTX_ERR_INVALID_ARG),
    (dict(scores=scores(softcap=2e38)), bd.CTX_ERR_INVALID_ARG),
    (dict(scores=scores(softcap=1e-40)), bd.CTX_ERR_INVALID_ARG),
    (dict(scores=scores(window=-1)), bd.CTX_ERR_INVALID_ARG),
    (dict(q=None), bd.CTX_ERR_INVALID_ARG),
    (dict(k_pages=None), bd.CTX_ERR_INVALID_ARG),
    (dict(v_pages=None), bd.CTX_ERR_INVALID_ARG),
    (dict(block_tables=None), bd.CTX_ERR_INVALID_ARG),
    (dict(seq_lens=None), bd.CTX_ERR_INVALID_ARG),
    (dict(out=None), bd.CTX_ERR_INVALID_ARG),
    (dict(q=18), bd.CTX_ERR_ALIGNMENT),
    (dict(k_pages=24), bd.CTX_ERR_ALIGNMENT),
    (dict(v_pages=20), bd.CTX_ERR_ALIGNMENT),
    (dict(out=24), bd.CTX_ERR_ALIGNMENT),
]


@pytest.mark.parametrize("kw,status", BOTH)
def test_scored_decode_refuses(lib, kw, status):
    assert lib.ctx_decode_attn_run_paged_scored(*decode_args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(total_q=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(max_q_len=-1), bd.CTX_ERR_INVALID_ARG),
    (dict(q_starts=None), bd.CTX_ERR_INVALID_ARG),
    (dict(q_lens=None), bd.CTX_ERR_INVALID_ARG),
])
def test_paged_prefill_refuses(lib, kw, status):
    assert lib.ctx_prefill_attn_run_paged(*prefill_args(**kw).values()) == status
    assert lib.ctx_decode_attn_last_error().decode()


def test_attention_over_nothing(lib):
    assert lib.ctx_decode_attn_run_paged_scored(*decode_args(num_seqs=0, q=None, out=None).values()) == bd.CTX_OK
    for kw in (dict(num_seqs=0), dict(max_q_len=0), dict(total_q=0)):
        assert lib.ctx_prefill_attn_run_paged(*prefill_args(q=None, out=None, **kw).values()) == bd.CTX_OK


def test_good_arguments_get_as_far_as_the_device(lib):
    """Without a GPU the device's query fails; with one, the handle's device is not the current one."""
    for rc in (lib.ctx_kv_append_run_paged(*append_args(rotary=rotary(q_norm=P16)).values()),
               lib.ctx_decode_attn_run_paged_scored(*decode_args(scores=scores(softcap=30.0, window=5)).values()),
               lib.ctx_prefill_attn_run_paged(*prefill_args(scores=scores(softcap=30.0, window=5)).values())):
        assert rc in (bd.CTX_ERR_HIP, bd.CTX_ERR_INVALID_ARG)
        assert "device" in lib.ctx_decode_attn_last_error().decode().lower()
