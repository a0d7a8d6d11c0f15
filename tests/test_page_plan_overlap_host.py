"""wam_page_plan refuses buffers that overlap, on the host: what is written may lie on nothing else (fake device addresses;
every call here is refused, none reaches a launch)."""
import ctypes as C
import itertools

import pytest

R, T, PAGES, WIDTH, STRIDE = 4, 50, 30, 8, 20
SIZES = dict(cache_len=R, new_len=R, held=R, n_free=1, table=(R - 1) * STRIDE + WIDTH, free_list=PAGES, held_out=R, n_free_out=1,
             q_start=R + 1, kv_len=R, slots=T, token_pos=T, status=4)
INPUTS = ("cache_len", "new_len", "held", "n_free")
PAIRS = [p for p in itertools.combinations(SIZES, 2) if not set(p) <= set(INPUTS)]


def call(**moved):
    import paper_2602_15922_amd as w
    b, L = w.binding, w.lib()
    at = {n: 4096 * (i + 1) for i, n in enumerate(SIZES)} | moved
    d = b.wam_page_plan_desc(R=R, T=T, page_size=16, n_pages=PAGES, max_pages=WIDTH, table_stride=STRIDE)
    return L.wam_page_plan(C.byref(d), *(at[n] for n in SIZES), None), L.wam_last_error().decode(), at


@pytest.mark.parametrize("a,b", PAIRS)
def test_every_pair(a, b):
    """b at a's first int, on a's last one, and ending on a's first one."""
    at = 4096 * (1 + list(SIZES).index(a))
    for where in (at, at + 4 * (SIZES[a] - 1), at - 4 * (SIZES[b] - 1)):
        status, says, _ = call(**{b: where})
        assert status == 1 and "overlap" in says, (where - at, says)
        assert all(x.replace("table", "block_table") in says for x in (a, b)), says


def test_the_next_turns_lengths_in_place():
    status, says, _ = call(kv_len=4096)  # cache_len's address
    assert status == 1 and "kv_len and cache_len overlap" in says


@pytest.mark.parametrize("row,col,n", [(0, 0, "held_out"), (1, WIDTH - 1, "status"), (2, 0, "slots"), (0, WIDTH, "slots"), (2, STRIDE - 1, "kv_len"),
                                       (3, WIDTH - 1, "n_free_out"), (0, STRIDE - 3, "status")])
def test_rows_of_a_wide_table(row, col, n):
    """Inside a row, and from the gap behind one into the next."""
    status, says, _ = call(**{n: 4096 * 5 + 4 * (row * STRIDE + col)})
    assert status == 1 and "block_table" in says and n in says, says
