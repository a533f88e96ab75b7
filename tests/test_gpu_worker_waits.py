"""The worker's rounds do not pass over a kernel that gave up waiting."""
import itertools

import pytest

from paper_2605_01989_b200 import binding as dblp
from paper_2605_01989_b200 import worker as wk

pytestmark = pytest.mark.gpu


def test_training_tells_of_a_wait_that_ran_out(monkeypatch):
    counts = itertools.count()
    monkeypatch.setattr(dblp, "dblp_wait_timeouts", lambda: next(counts))
    with pytest.raises(RuntimeError, match="gave up"):
        wk.train(2)


def test_training_does_not_mind_what_ran_out_before(monkeypatch):
    monkeypatch.setattr(dblp, "dblp_wait_timeouts", lambda: 3)
    assert len(wk.train(2)) == 2
