"""The rule for the columns of the attention of drafted trees, on the host."""
import pytest

import tree_form


def test_ctas_of_an_sm_follow_the_prefix():
    """A prefix's scores lie in shared memory: two CTAs of 32 or 64 columns share an SM beside a short one only (the sizes are asserted where the kernel is)."""
    ctas = lambda columns, own, n_prefix: tree_form.rule().ctas(columns, own, n_prefix)
    for own, n32, n64 in ((0, 56, 24), (1, 24, 12)):
        assert [ctas(c, own, 4) for c in (32, 64, 128)] == [2, 2, 1]
        assert (ctas(32, own, n32), ctas(32, own, n32 + 1)) == (2, 1)
        assert (ctas(64, own, n64), ctas(64, own, n64 + 1)) == (2, 1)
        assert [ctas(c, own, 64) for c in (32, 64, 128)] == [1, 1, 1]


@pytest.mark.parametrize("own", [0, 1])
def test_a_long_prefix_changes_the_choice(own):
    """One item's worth of CTAs to an SM: what two rounds of CTAs would take counts as two rounds. 16 trees of 16 rows at 4000 keys, 32 heads on 8: with 28 prefixed keys 32
    columns take 56 us and 64 take 74 (static steps; own steps 80 and 77)."""
    at = lambda n_prefix: tree_form.columns(own, n_prefix, 16, 8, 4, 16, 4000)
    assert at(4) == 64
    assert at(28) == (128 if own else 32)
    assert at(64) == 128


def test_a_window_bounds_what_is_counted():
    assert tree_form.columns(0, 4, 16, 8, 4, 33, 30000, 256, 4) == tree_form.columns(0, 4, 16, 8, 4, 33, 256 + 4 + 384, 0, 0)


def test_every_number_of_columns_is_taken_by_some_call():
    for own in (0, 1):
        for G in range(1, 9):
            for want in (32, 64, 128):
                assert tree_form.call_for(want, own, 4, 3, 2, G, 20, 700) is not None
                assert tree_form.call_for(want, own, 4, 3, 2, G, 20, 700, 300, 20) is not None
