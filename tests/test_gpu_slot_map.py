"""Slot maps of more rows than a step's, into outputs that begin anywhere: every entry of the map is
written, and nothing beside it.  Whole numbers: equality."""
import numpy as np
import pytest
import torch

from paper_2608_21541_gb300 import certkv as ck
from test_gpu_pages import PAGE, ints, map_of, random_store

pytestmark = pytest.mark.gpu
FILL = -77  # what the buffer around a map holds; no entry is that


def mapped_into(st, T, at, rows, start, batch):
    """The map in a view `at` entries into a larger buffer, and what the call left around it."""
    n = st.units * T
    buf = torch.full((n + 16,), FILL, dtype=torch.int32, device="cuda")
    assert buf.data_ptr() % 16 == 0
    view = buf[at:at + n].view(st.units, T)
    got, pos = ck.certkv_slot_map(st, T, rows=None if rows is None else ints(rows),
                                  start=None if start is None else ints(start), batch=batch, slots=view)
    assert got.data_ptr() == view.data_ptr()
    return view.cpu().numpy(), pos.cpu().numpy(), torch.cat((buf[:at], buf[at + n:]))


# both sides of the step's kernel's end, one block's rows and several, multiples of 4 and not
ROWS = [511, 512, 513, 514, 515, 516, 16383, 16384, 16385, 16386, 16387, 32768, 40001]


@pytest.mark.parametrize("T", ROWS)
@pytest.mark.parametrize("given", [False, True])
def test_maps_into_any_place(T, given):
    units, batch = 6, 3
    max_pages = 4 + T // PAGE
    st, rng = random_store(units, max_pages, 2 * units * max_pages, T, share=1.0)
    st.counts.copy_(ints(rng.integers(0, 3 * PAGE, units)))
    st.table[2, 1] = -1  # no page in the middle of a segment
    rows = [T, T - 3, T // 2] if given else None
    start = rng.integers(-5, 4 * PAGE, units) if given else None
    want, positions = map_of(st, T, rows, start, batch=batch)
    for at in (0, 1, 2, 3, 4, 7):
        got, pos, around = mapped_into(st, T, at, rows, start, batch)
        np.testing.assert_array_equal(got, want, err_msg=f"{at} entries in")
        np.testing.assert_array_equal(pos, positions)
        assert (around == FILL).all(), at


@pytest.mark.parametrize("at", [1, 2, 3])
def test_a_long_prompt_of_one_segment(at):
    T = 131072
    st, _ = random_store(1, T // PAGE, 2 * T // PAGE, 9, share=1.0)
    st.counts.zero_()
    want, _ = map_of(st, T)
    got, _, around = mapped_into(st, T, at, None, None, 1)
    np.testing.assert_array_equal(got, want)
    assert (around == FILL).all()
