"""Arrays of the calls on pages that a call writes and that share memory with others are refused before the
device is asked for anything; neighbours in one buffer are not."""
import pytest

from paper_2609_36608_amd import binding as bd
from test_kv_pages_abi_cpu import compact_args, fork_args, resize_args

SEQS, WIDTH, PAGES, ROWS = 2, 4, 8, 9


@pytest.fixture(scope="module")
def lib():
    return bd.load_library()


def laid_out(at=4096, **sizes):
    """Addresses of arrays of 32-bit values right behind each other."""
    out = {}
    for name, values in sizes.items():
        out[name] = at
        at += 4 * values
    return out


FORK = dict(block_tables=SEQS * WIDTH, seq_lens=SEQS, parents=SEQS, page_refs=PAGES)
RESIZE = dict(workspace=2 * SEQS + PAGES, copies=2 * SEQS, block_tables=SEQS * WIDTH, seq_lens=SEQS, new_lens=SEQS,
              granted=SEQS, page_refs=PAGES)
COMPACT = dict(block_tables=SEQS * WIDTH, seq_lens=SEQS, q_starts=SEQS, q_lens=SEQS, keep=ROWS, keep_lens=SEQS,
               new_lens=SEQS)
CACHES = dict(k_pages=1 << 20, v_pages=(1 << 20) + PAGES * 16 * 8 * 128 * 2)
CALLS = {"fork": ("ctx_kv_fork_run_paged", fork_args, FORK, {}),
         "resize": ("ctx_kv_resize_run_paged", resize_args, RESIZE, {}),
         "compact": ("ctx_kv_compact_run_paged", compact_args, COMPACT, CACHES)}


def run(lib, call, **kw):
    name, args, sizes, more = CALLS[call]
    rc = getattr(lib, name)(*args(**(laid_out(**sizes) | more | kw)).values())
    return rc, lib.ctx_decode_attn_last_error().decode()


@pytest.mark.parametrize("call", CALLS)
def test_neighbours_are_taken(lib, call):
    rc, message = run(lib, call)
    assert "overlap" not in message and (rc == bd.CTX_ERR_HIP or "device" in message)  # the next check


def pairs():
    for call, written in (("fork", ("block_tables", "seq_lens", "page_refs")),
                          ("resize", ("block_tables", "page_refs", "copies", "granted", "workspace")),
                          ("compact", ("new_lens",))):
        sizes = CALLS[call][2]
        for x in written:
            for y in sizes:
                if y != x:
                    yield call, x, y


@pytest.mark.parametrize("call,x,y", pairs())
def test_overlaps_are_refused(lib, call, x, y):
    """x's first or last value is y's last or first."""
    sizes = CALLS[call][2]
    step = 16 if "workspace" in (x, y) else 8 if "copies" in (x, y) else 4  # bytes, aligned
    far = {name: (1 << 16) + 4096 * i for i, name in enumerate(sizes)} | {y: 1 << 15}
    for place in (far[y] + 4 * sizes[y] - step, far[y] - 4 * sizes[x] + step):
        rc, message = run(lib, call, **(far | {x: place // step * step}))
        assert rc == bd.CTX_ERR_INVALID_ARG and "overlap" in message, (x, y, place, message)


def test_lengths_in_place(lib):
    at = laid_out(**RESIZE)
    for name in ("seq_lens", "new_lens"):
        rc, message = run(lib, "resize", granted=at[name])
        assert "overlap" not in message, message
    rc, message = run(lib, "resize", granted=at["seq_lens"], new_lens=at["seq_lens"])
    assert "overlap" not in message, message
    rc, message = run(lib, "resize", granted=at["seq_lens"], new_lens=at["seq_lens"] + 4)
    assert rc == bd.CTX_ERR_INVALID_ARG and "overlap" in message


def test_caches(lib):
    for k, v in ((CACHES["k_pages"],) * 2, (CACHES["k_pages"], CACHES["v_pages"] - 256)):
        rc, message = run(lib, "compact", k_pages=k, v_pages=v)
        assert rc == bd.CTX_ERR_INVALID_ARG and "k_pages and v_pages" in message
