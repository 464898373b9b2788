"""The stack with attention layers among the linear ones: served token by token and as longer prompts."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# Both ways round the same values, as in test_gpu_linear_layers (fp32 1e-4, bf16 0.05, fp16 0.05 / 8). A cached
# value that lies at a border of its format may fall to either side of it: in fp32 about one in 2^8 * 1e-4 of
# 16 bits does, by 2^-8 of itself, 2^-8 * sqrt(0.026) = 6e-4 of the norm at most; codes of 8 bits have steps of
# absmax / 127, some 3 / 127 of the norm.
@pytest.mark.parametrize("dtype,cache,bound", [("float32", "bfloat16", 1e-4 + 6e-4), ("float16", "float16", 0.05 / 8),
                                               ("bfloat16", "bfloat16", 0.05), ("bfloat16", "int8", 0.05 + 3 / 127)])
@pytest.mark.parametrize("size", [dict(requests=3, tokens=9, longest=90, layers=2, hk=2, hv=4, hidden=256, attention_every=2),
                                  dict(requests=12, tokens=5, longest=600, layers=4, hk=2, hv=8, hidden=512, attention_every=2),
                                  dict(requests=5, tokens=3, longest=70, layers=3, hk=1, hv=12, hidden=256, attention_every=1)],
                         ids=["few", "many", "attention-only"])
def test_tokens_continue_prompts(size, dtype, cache, bound):
    from paper_2609_38169_gb300 import linear_layers
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    r = linear_layers.serve(dtype=getattr(torch, dtype), cache=cache, **size)
    assert r["device_error"] == 0
    assert r["outputs_apart"] <= bound, r
    if size["attention_every"] > 1:
        assert r["states_apart"] <= bound, r
