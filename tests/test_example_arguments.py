"""The example's own refusals, before anything runs."""
import sys
from pathlib import Path

import pytest

sys.path.insert(0, str(Path(__file__).resolve().parents[1] / "examples"))
import endless_chat  # noqa: E402


@pytest.mark.parametrize("name", ["conversations", "prompt", "forks", "steps", "layers"])
@pytest.mark.parametrize("n", [0, -3])
def test_nothing_to_do_is_refused(monkeypatch, name, n):
    def no_gpu():
        raise AssertionError("past the checks")
    monkeypatch.setattr(endless_chat.pda, "load", no_gpu)
    with pytest.raises(ValueError, match=name):
        endless_chat.run(**{name: n})
    with pytest.raises(AssertionError):
        endless_chat.run(**{name: 1})
