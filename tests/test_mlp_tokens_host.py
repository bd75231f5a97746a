"""The dense-layer example on tokens without a GPU: what it refuses before anything is allocated."""
import pytest

from paper_2406_05546_amd import mlp


@pytest.mark.parametrize("bad", [dict(vocab=-1), dict(vocab=10, context=0), dict(vocab=10, context=3)])
def test_servers_that_are_refused(bad):
    args = dict(widths=[4, 3], n_versions=1, capacity=1)
    args.update(bad)
    with pytest.raises(ValueError):
        mlp.MlpServer(**args)
