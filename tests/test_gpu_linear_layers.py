"""The stack of linear-attention layers: served token by token and as longer prompts."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# Both ways round the same values. fp32: errors of some hundred u = 2^-24 a layer, through a few
# layers of gain about one: 1e-4. 16 bits: some ten roundings of half a unit (2^-8 or 2^-11) a
# layer, adding up as squares: 4 layers of them are below 2^-8 * sqrt(40) * 2 (the gain) = 0.05.
@pytest.mark.parametrize("dtype,bound", [("float32", 1e-4), ("bfloat16", 0.05), ("float16", 0.05 / 8)])
@pytest.mark.parametrize("size", [dict(requests=3, tokens=9, longest=90, layers=2, hk=2, hv=4, hidden=256),
                                  dict(requests=20, tokens=5, longest=1500, layers=4, hk=2, hv=8, hidden=512)], ids=["few", "many"])
def test_tokens_continue_prompts(size, dtype, bound):
    from paper_2609_38169_gb300 import linear_layers
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    r = linear_layers.serve(dtype=getattr(torch, dtype), **size)
    assert r["device_error"] == 0
    assert r["states_apart"] <= bound and r["outputs_apart"] <= bound, r
