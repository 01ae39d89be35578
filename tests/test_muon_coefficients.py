"""Coefficients of the steps as the binding takes them (CPU)."""

import pytest

ROWS = [(3.5, -4.5, 2.0), (3.0, -4.0, 2.0)]
FLAT = [x for r in ROWS for x in r]


@pytest.mark.parametrize("given", [ROWS, tuple(ROWS), [list(r) for r in ROWS], tuple(list(r) for r in ROWS)])
def test_one_triple_for_each_step_in_any_sequence(given):
    from paper_2609_30656_gb300 import muon
    for _ in range(2):  # the second time from what was kept, where something was
        assert list(muon._coefficients(given, 2)) == FLAT


def test_one_triple_for_all_steps():
    from paper_2609_30656_gb300 import muon
    for given in (ROWS[0], list(ROWS[0])):
        assert list(muon._coefficients(given, 3)) == list(ROWS[0]) * 3


class Value:
    """A number that changes, as a tensor of one value does: equal and hashed by identity."""

    def __init__(self, x):
        self.x = x

    def __float__(self):
        return self.x


def test_values_that_change_are_read_in_every_call():
    from paper_2609_30656_gb300 import muon
    v = Value(3.5)
    for given in (((v, -4.5, 2.0),), (v, -4.5, 2.0)):
        for x in (3.5, 3.25):
            v.x = x
            assert list(muon._coefficients(given, 1)) == [x, -4.5, 2.0]
