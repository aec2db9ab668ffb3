"""The hand-over of a split model's caches, with all of the serving operators as they are used together."""
import pytest

from paper_2511_04002_amd import serve

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 128)])
def test_receiver_goes_on_where_the_sender_was(dtype, heads):
    q_heads, kv_heads, dim = heads
    r = serve.run(requests=5, prompt=150, layers=2, steps=20, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype)
    assert r["tokens_sent"] == 30 + 60 + 90 + 120 + 150
    assert 0 < r["sent_bytes"] < r["cache_bytes"]
    # what is sent is within the budget (1 % of a row's RMS) of the sender's cache; the receiver's own 8 bits add half a step of
    # 1/127 of a block's largest, about 1 % of the RMS; both act on the attention of two layers
    assert 0 <= r["relative_difference"] < 0.08


def test_one_request_and_one_token():
    r = serve.run(requests=1, prompt=1, layers=1, steps=3, q_heads=4, kv_heads=1, dim=64, dtype="f16")
    assert r["tokens_sent"] == 1 and r["relative_difference"] < 0.08
