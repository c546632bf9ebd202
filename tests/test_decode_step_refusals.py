"""What step.DecodeStep refuses, before the calls that it makes have changed anything (CPU)."""
import pytest
import torch

import mx4_reference as R


@pytest.fixture(scope="module")
def mla():
    from paper_2609_07008_amd import mla as m
    return m


def _step(**over):
    from paper_2609_07008_amd.step import DecodeStep
    a = {**dict(geom=R.geom(16), n_seqs=2, n_q=1, max_pages=3, page_rows=64, d_out=64), **over}
    return DecodeStep(**a, device="cpu")


# more inputs than W_b takes, no channel or too many, types that it does not write
@pytest.mark.parametrize("over", [dict(geom=R.geom(16, d_model=32768)), dict(geom=R.geom(16, d_model=16448)), dict(d_out=0), dict(d_out=-3),
                                  dict(d_out=2 ** 24 + 1), dict(d_out=2 ** 25), dict(y_dtype=torch.float16), dict(y_dtype=torch.float64),
                                  dict(y_dtype=None)])
def test_refused_where_it_is_made(mla, over, monkeypatch):
    def no_buffer(*a, **k):
        raise AssertionError("a buffer was made")
    for f in ("empty", "arange", "full"):
        monkeypatch.setattr(torch, f, no_buffer)
    with pytest.raises(mla.MlaError):
        _step(**over)


@pytest.mark.parametrize("over", [dict(), dict(geom=R.geom(16, d_model=16384)), dict(d_out=1), dict(y_dtype=torch.float32)])
def test_made_at_the_edges(mla, over):
    st = _step(**over)
    assert tuple(st.y.shape) == (2, over.get("d_out", 64))
