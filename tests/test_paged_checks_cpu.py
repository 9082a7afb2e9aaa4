"""More refusals of the calls over paged caches that need no GPU."""
import pytest

from paper_2609_36608_amd import binding as bd

from test_paged_abi_cpu import decode_args, lib, prefill_args, scores  # noqa: F401


@pytest.mark.parametrize("flags,status", [(2, bd.CTX_ERR_INVALID_ARG), (0x80000001, bd.CTX_ERR_INVALID_ARG), (0, None),
                                          (bd.CTX_SCORES_SPLIT_P, None)])
def test_unknown_score_flags_are_refused(lib, flags, status):  # noqa: F811
    kw = dict(scores=scores(flags=flags))
    for rc in (lib.ctx_decode_attn_run_paged_scored(*decode_args(num_seqs=0, **kw).values()),
               lib.ctx_prefill_attn_run_paged(*prefill_args(num_seqs=0, **kw).values())):
        assert rc == (bd.CTX_OK if status is None else status)


@pytest.mark.parametrize("window", [2 ** 31, 2 ** 32 + 5, 2 ** 63, -2 ** 31 - 1])
def test_windows_that_32_bits_would_wrap_are_refused(window):
    with pytest.raises(ValueError):
        bd._scores_struct(bd.AttnScores(window=window), 0, 8, 1, 1)


@pytest.mark.parametrize("softcap", [1e-46, 5e-324, -1e-50])
def test_caps_that_a_float_would_make_none_are_refused(softcap):
    with pytest.raises(ValueError):
        bd._scores_struct(bd.AttnScores(softcap=softcap), 0, 8, 1, 1)
