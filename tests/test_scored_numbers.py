"""Numbers of the binding that the library takes as 32 bits: refused where they do not fit."""
import pytest
import torch

from paper_2403_20137_amd import kvbfp


@pytest.mark.parametrize("window", [2 ** 32 + 5, 2 ** 32, 2 ** 31, -2 ** 31 - 1])
def test_windows(window):
    with pytest.raises(ValueError, match="window"):
        kvbfp.make_score_rule(window=window)


def test_windows_that_fit():
    assert kvbfp.make_score_rule(window=2 ** 31 - 1).window == 2 ** 31 - 1 and kvbfp.make_score_rule(window=-1).window == -1


@pytest.mark.parametrize("name", ["n_first", "n_recent"])
def test_tokens_that_stay(name, monkeypatch):
    monkeypatch.setattr(kvbfp, "_dev_ptr", lambda t, dtype=None: None if t is None else t.data_ptr())
    z = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    cache = kvbfp.Cache(kvbfp.make_layout(128, 32, 4, 2, 3, 512), z(1), z(1), z(1), z(1))
    numbers = {**dict(n_first=4, n_recent=10), name: 2 ** 32 + 1}
    with pytest.raises(ValueError, match=name):
        kvbfp.evict(cache, cache, torch.zeros(3, 2, 512), 512, 100, kept=torch.zeros(3, 2, 100, dtype=torch.int32),
                    new_len=torch.zeros(3, dtype=torch.int32), stream=0, **numbers)
