"""The operators of the cache together, behind and before the quantized projections."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_prompts_and_decoding_through_a_layer_match_attention_without_a_cache():
    """What the 8 bits cost: keys and values carry a relative error of up to 2^-4 per element (2^-5.2 on average over a binade),
    which an average over keys does not raise; a misplaced token or page gives an error of order 1."""
    from paper_2501_04052_amd import cached_attention
    assert cached_attention.run(prompts=(5, 70, 1), steps=6) < 2.0 ** -4
    assert cached_attention.run(hidden=512, q_heads=12, kv_heads=4, head_dim=64, prompts=(130, 33), steps=3, page=16) < 2.0 ** -4


def test_a_pool_without_room_refuses_the_step():
    from paper_2501_04052_amd.cached_attention import PagePool
    pool = PagePool(3, 2, 64, page=16)
    pool.step([16, 17])
    with pytest.raises(RuntimeError):
        pool.step([1, 0])
    with pytest.raises(RuntimeError):
        PagePool(30, 2, 64, page=16).step([65, 0])
    plan, known = pool.step([0, 1])
    assert known == dict(max_new=1, max_len=18) and plan.slots.tolist() == [2 * 16 + 1]
