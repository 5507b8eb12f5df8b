"""The preference step among workers that lie: it runs, and honest copies of a file agree bit for bit."""
import pytest

from paper_2010_04902_b200 import worker_step as ws

pytestmark = pytest.mark.gpu


def test_preference_with_liars():
    losses = ws.tune(2, 3, "preference", same_bits=True)
    assert len(losses) == 2 and all(abs(v) < 1e3 for v in losses)
