"""The page tables without a GPU: tokens taken back (refusals, the operator's fake implementation, the plain form's invariants) and rows that overlap."""
import random

import pytest

torch = pytest.importorskip("torch")

import cache_back  # noqa: E402
import paper_2408_11743_amd as mk  # noqa: E402
from test_cache_cpu import ALIGN, FAKE, PAGES, SHAPE, WS, invariants, state, status  # noqa: E402


def test_back_is_optional_and_aligned():
    assert status("pages", back=FAKE + 2) == ALIGN
    assert status("pages", back=FAKE, workspace_bytes=8) == WS == status("pages", back=None, workspace_bytes=8)
    with pytest.raises(mk.MarlinError):
        mk.marlin_assign_pages(**{**PAGES, "workspace_bytes": 8})


def test_fake_of_tokens_taken_back():
    def ints(*shape):
        return torch.empty(*shape, dtype=torch.int32, device="meta")
    starts, slots = torch.ops.marlin_mi355x.assign_pages(ints(3, 4), ints(3), ints(3), ints(9), ints(1), 16, 11, 0, 0, ints(3))
    assert starts.shape == (4,) and slots.shape == (11,)


def test_pages_reference_with_tokens_taken_back():
    """Whatever is taken back: every page is in one place once, and lengths are what is left and what is new."""
    rng = random.Random(3)
    for _ in range(300):
        table, lengths, new, free, count = state(rng, rng.randrange(1, 9))
        back = torch.tensor([rng.choice([-5, 0, 0, 1, 3, 16, 40, 1000]) for _ in lengths], dtype=torch.int32)
        tokens, window = rng.choice([0, 5, 60, 1000]), rng.choice([None, None, 1, 16, 40])
        after = cache_back.assign_pages(table, lengths, new, free, count, 16, tokens, window, rng.choice([0, 1, 20]), back)
        short = cache_back.take_back(table, lengths, free, count, 16, back)
        assert torch.equal(short[1], (lengths - back.clamp(min=0)).clamp(min=0))
        named = (short[0] >= 0).sum(1)
        assert (named == (short[1] + 15) // 16).all()
        invariants((short[0], short[1], short[2], short[3], new), after, 16, tokens)
        assert int(short[3]) + int(named.sum()) == int(count) + int((table >= 0).sum())


def test_rows_of_a_table_that_overlap_are_refused():
    """Both would be written."""
    for row in (0, 1, PAGES["width"] - 1):
        assert status("pages", table_row=row, workspace_bytes=8) == SHAPE
        assert status("pages", table_row=row, B=1, workspace_bytes=8) == WS
    assert status("pages", table_row=PAGES["width"], workspace_bytes=8) == WS
