"""The hand-over of a split model's caches held in 4 bits, with tokens of pictures, with all of the serving operators as they are
used together."""
import pytest

from paper_2511_04002_amd import cache, serve

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 128), (4, 1, 256)])
@pytest.mark.parametrize("images", [False, True])
def test_receiver_goes_on_where_the_sender_was(dtype, heads, images):
    q_heads, kv_heads, dim = heads
    r = serve.run(requests=5, prompt=150, layers=2, steps=20, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, cache_bits=4, images=images)
    assert r["tokens_sent"] == 30 + 60 + 90 + 120 + 150
    assert 0 < r["sent_bytes"] < r["cache_bytes"]
    # what is sent is what the sender's cache stands for, coded in 4 to 8 bits a token within 1 % of a row's RMS, and the receiver codes
    # it again in 4 bits: 0.112 of the RMS of normal data where values fall anew, but nearly all fall back to where they were
    assert 0 <= r["relative_difference"] < 0.15


def test_pictures_in_8_bits_and_one_token():
    r = serve.run(requests=3, prompt=150, layers=1, steps=3, q_heads=4, kv_heads=1, dim=64, dtype="f16", images=True)
    assert r["relative_difference"] < 0.08
    r = serve.run(requests=1, prompt=1, layers=1, steps=3, q_heads=4, kv_heads=1, dim=64, dtype="f16", cache_bits=4)
    assert r["tokens_sent"] == 1 and r["relative_difference"] < 0.15


@pytest.mark.parametrize("bits", [8, 4])
def test_what_is_sent_is_set_beside_what_the_caches_hold(bits):
    r = serve.run(requests=4, prompt=128, layers=2, steps=1, q_heads=8, kv_heads=2, dim=128, dtype="bf16", cache_bits=bits)
    tokens = 32 + 64 + 96 + 128                              # whole blocks of 16: as many bytes as a cache of so many has
    c = cache.Cache(tokens // 16, 16, 8, 2, 128, "bf16", 8, bits=bits)
    sizes = cache.tsq_cache_memory_sizes(c.handle)
    assert r["tokens_sent"] == tokens and r["held_bytes"] == 2 * 2 * (sizes.code_bytes + sizes.scale_bytes)
    assert r["cache_bytes"] == 2 * 2 * tokens * 2 * 128 * 2
    assert 0 < r["sent_bytes"] < r["cache_bytes"]
