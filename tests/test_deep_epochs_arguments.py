"""Defaults of `deep_epochs.py`'s command line."""
import pytest


@pytest.mark.parametrize("argv,lr", [([], 0.5), (["--ff", "2"], 0.5), (["--ff", "2", "--adamw", "8bit"], 1e-3), (["--adamw", "32bit"], 1e-3),
                                     (["--adamw", "8bit", "--lr", "0.25"], 0.25), (["--lr", "0"], 0.0)], ids=str)
def test_the_learning_rate_goes_by_the_optimizer(argv, lr):
    from deep_epochs import arguments
    assert arguments(argv).lr == lr
