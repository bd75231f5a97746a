"""The dense-layer example without a GPU: what it refuses before anything is allocated."""
import pytest

from paper_2406_05546_amd import mlp


@pytest.mark.parametrize("bad", [dict(widths=[4]), dict(widths=[4, 0]), dict(n_versions=0), dict(capacity=0), dict(activation="tanh")])
def test_servers_that_are_refused(bad):
    args = dict(widths=[4, 3], n_versions=1, capacity=1)
    args.update(bad)
    with pytest.raises(ValueError):
        mlp.MlpServer(**args)
