"""Host logic of grouped rollouts: the tables of shared pages, and what the toggle is given.  No GPU."""
from unittest import mock

import numpy as np
import pytest

from paper_2606_18967_amd import rollout


def test_grouped_tables():
    table, gid, n = rollout.grouped_tables(6, 3, 2, 130, 300, 64)
    assert table.shape == (8, 5) and gid.tolist() == [0, 0, 0, 1, 1, 1, 1, 1]
    assert (table[:3, :2] == table[0, :2]).all() and (table[3:, :2] == table[3, :2]).all()
    own = table[:, 2:].ravel().tolist() + table[0, :2].tolist() + table[3, :2].tolist()
    assert sorted(own) == list(range(n))                          # no page twice but the shared ones
    with pytest.raises(ValueError):
        rollout.grouped_tables(7, 3, 0, 130, 300, 64)


def test_decode_of_groups_prices_a_prompt_once():
    seen = []

    def fake_toggle(m, B, S, tau, gamma, eps, on):
        seen.append((B, S))
        return 0

    live = {"n": 4}

    def ar():
        return np.ones(live["n"], dtype=np.int64)

    def compact(keep):
        live["n"] = int(keep.sum())

    with mock.patch.object(rollout.sdrl, "toggle", fake_toggle):
        rollout.decode(np.array([1, 2, 3, 3]), 100, "toggle", 5, 5.0, None, 0.05, ar, None, compact, group=2)
    assert seen == [(4, 50.0), (3, 100 * 2 / 3 + 1.0), (2, 50.0 + 2.0)]


@pytest.mark.parametrize("B,group", [(6, 0), (6, 4), (2, 3), (6, -1)])
def test_batches_are_whole_groups(B, group):
    with pytest.raises(ValueError, match="whole groups"):
        rollout.Rollout({}, B, 100, 20, group=group)
