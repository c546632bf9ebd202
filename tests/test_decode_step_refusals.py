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


BF16 = torch.bfloat16
W_O = (1, 16 * 512, 256)


@pytest.mark.parametrize("w_o", [None, torch.zeros(W_O), torch.zeros((1, 16 * 512, 128), dtype=BF16), torch.zeros((1, 8 * 512, 256), dtype=BF16),
                                 torch.zeros((1, 16 * 512, 512), dtype=BF16)[..., :256], torch.zeros(0, dtype=BF16)])
def test_weight_of_the_o_proj(mla, w_o, monkeypatch):
    """Its address alone reaches the library: type, size and layout are checked here."""
    st = _step()
    monkeypatch.setattr(mla, "_device", lambda: -1)      # host tensors count as on the current device
    monkeypatch.setattr(mla, "sliced_oproj_add_planned", lambda *a: pytest.fail("reached the library"))
    with pytest.raises(mla.MlaError) as e:
        st.oproj(w_o)
    assert "w_o" in str(e.value)


def test_weight_of_the_o_proj_on_another_device(mla, monkeypatch):
    st = _step()
    monkeypatch.setattr(mla, "_device", lambda: 0)
    with pytest.raises(mla.MlaError):
        st.oproj(torch.zeros(W_O, dtype=BF16))


@pytest.mark.parametrize("shape", [W_O, (16 * 512, 256), (16, 512, 256)])
def test_weight_of_the_o_proj_in_any_shape_of_its_size(mla, shape, monkeypatch):
    st, got = _step(), []
    monkeypatch.setattr(mla, "_device", lambda: -1)
    monkeypatch.setattr(mla, "sliced_oproj_add_planned", lambda *a: got.append(a))
    st.oproj(torch.zeros(shape, dtype=BF16))
    assert len(got) == 1
