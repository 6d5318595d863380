"""Lengths, pages and slots next to the ends of their types."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("page", [1, 2, 16, 2 ** 30, MOST])
@pytest.mark.parametrize("max_new", [3, 5000])                       # slots by the first kernel, and by the second
@pytest.mark.parametrize("length", [MOST, MOST - 1, 2 ** 30 - 1, 2 ** 30])
def test_positions_beyond_31_bits(spec, length, max_new, page):
    """Positions from `length` on may pass 2^31: they lie behind every page, or on the last one, never before the table."""
    width, held = 4, 3
    lens, table, pages = i32([5, length, 2]), i32([[7, 8, 9, -1]] * 3), i32([held] * 3)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = spec.spec_page_tables(lens, None, table, pages, i32([1, 2]), i32([2]), page, max_new=max_new, err_workspace=err)
    held, count, short, want = [3, 3, 3], 2, False, []
    for b, n in enumerate((5, length, 2)):
        pages_wanted = -(-(n + max_new) // page)
        if pages_wanted > width:
            short = True
        elif pages_wanted > held[b]:
            held[b], count = pages_wanted, count - (pages_wanted - held[b])
    row = table.tolist()
    for b, n in enumerate((5, length, 2)):
        at = [n + j for j in range(max_new)]
        want.append([row[b][p // page] * page + p % page if p // page < held[b] else -1 for p in at])
    assert count >= 0 and pages.tolist() == held and slots.tolist() == want
    assert spec.spec_poll_error(err) == (spec.SPEC_ERR_PAGES if short else spec.SPEC_OK)
