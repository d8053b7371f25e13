"""The attention kernel's failure path: a block whose values never arrive gives up after a short limit, says so and leaves the
cache usable."""
import pytest
import torch

import paper_2604_17701_b200 as wisv
from test_gpu_paged import build, dev

pytestmark = pytest.mark.gpu

SHAPES = {
    # n_new, kv_len, H, kv, d, page, dtype, the block that gets no values
    "shared items": ([9], [3000], 32, 8, 128, 16, "bf16", 3),
    "batch": ([9, 1, 30], [900, 40, 3000], 32, 8, 128, 16, "bf16", 0),
    "pairs of row tiles": ([700], [2000], 8, 2, 128, 64, "fp16", 5),
    "head size 64": ([70, 3], [2500, 900], 14, 2, 64, 32, "bf16", 1),
    "whole items": ([1] * 200, [700] * 200, 8, 8, 64, 16, "fp16", 17),
}


def setup(name):
    n_new, kv_len, H, kv, d, page, dtype, block = SHAPES[name]
    cache, q, kp, vp, q_off = build(n_new=n_new, kv_len=kv_len, H=H, kv=kv, d=d, page=page, dtype=dtype, seed=4)
    args = (kp, vp, dev(kv_len))
    kw = dict(B=len(n_new), max_new=max(n_new), q_off=dev(q_off))
    return cache, lambda x=1.0: cache.attend(q * x, *args, **kw), block


@pytest.mark.parametrize("name", SHAPES)
def test_waits_give_up_and_the_cache_stays_usable(name):
    cache, attend, block = setup(name)
    first = attend()
    assert cache.device_error() == 0
    cache.debug_waits(2_000_000, block)                            # about 1 ms
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    attend()
    end.record()
    assert cache.device_error() == 1                               # reported ...
    assert cache.device_error() == 0                               # ... and cleared
    assert begin.elapsed_time(end) < 500                           # everything in flight was waited for, nothing else
    cache.debug_waits(2_000_000)                                   # the limit alone does not bother a block that gets its values
    assert torch.equal(attend(), first) and cache.device_error() == 0
    cache.debug_waits()
    assert torch.equal(attend(), first) and cache.device_error() == 0
    cache.close()


def test_refusals():
    cache, _, _ = setup("batch")
    for limit, block in ((5_000_000_000, -1), (0, -2)):
        with pytest.raises(wisv.WisvError) as e:
            cache.debug_waits(limit, block)
        assert e.value.code == -1
    cache.close()


@pytest.mark.parametrize("name", SHAPES)
def test_calls_after_a_time_out_are_right_before_it_is_read(name):
    """Graph replays cannot read the error word: arrivals that a failed call left behind must not count in the next ones."""
    cache, attend, block = setup(name)
    inputs = [1.0, -2.0, 0.5, 3.0]                                 # other queries every time, so that stale partials show
    want = [attend(x) for x in inputs]
    assert cache.device_error() == 0
    for fails in (1, 2, 1):                                        # twice in a row as well
        cache.debug_waits(2_000_000, block)
        for _ in range(fails):
            attend(1.5)
        cache.debug_waits()
        for x, y in zip(inputs, want):
            assert torch.equal(attend(x), y), (fails, x)
    assert cache.device_error() == 1                               # still reported
    assert torch.equal(attend(2.0), attend(2.0)) and cache.device_error() == 0
    cache.close()
