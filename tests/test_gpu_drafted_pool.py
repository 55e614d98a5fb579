"""What the decoding loop refuses about pools, forks and prompts, before anything has changed."""
import pytest
import torch

pytestmark = pytest.mark.gpu
PROMPTS = [[3, 1, 4, 1, 5], [7] * 33]


def _decoder(**kw):
    from paper_2607_04031_b200.drafted import Decoder
    return Decoder(**{**dict(requests=4, cache="e2m1", page_tokens=16, room=256), **kw})


def _state(d):
    kept = [d.start, d.page_table, *d.pool] + ([] if d.last is None else [d.last]) + (list(d.tables._tensors) if d.tables is not None else [])
    return [t.clone() for t in kept]


def _unchanged(d, before):
    after = _state(d)
    assert len(after) == len(before)
    assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(after, before))


@pytest.mark.parametrize("call", [lambda d: d.fork(2), lambda d: d.compact(), lambda d: d.generate(PROMPTS, 4, 2, 2, samples=2)])
@pytest.mark.parametrize("filled", [False, True])
def test_forks_and_compaction_need_a_pool(call, filled):
    d = _decoder()
    if filled:
        d.prefill(PROMPTS * 2)
    before = _state(d)
    with pytest.raises(ValueError, match="pool"):
        call(d)
    _unchanged(d, before)


def test_a_fork_needs_something_to_continue():
    d = _decoder(pool_pages=40)
    before = _state(d)
    with pytest.raises(ValueError, match="prefill"):
        d.fork(2)
    _unchanged(d, before)


@pytest.mark.parametrize("call", [lambda d: d.fork(2), lambda d: d.generate(PROMPTS, 4, 2, 2, samples=2)])
def test_requests_that_hold_pages_are_not_forked_to(call):
    from paper_2607_04031_b200 import binding as tl
    d = _decoder(pool_pages=80)
    made, _ = d.generate(PROMPTS, 4, 2, 2, samples=2)
    assert [len(m) for m in made] == [4] * 4
    before = _state(d)
    with pytest.raises(ValueError, match="hold"):
        call(d)
    _unchanged(d, before)
    tl.device_status()
    d.step(2, 2)                                             # they go on as before
    tl.device_status()


@pytest.mark.parametrize("samples", [0, -1])
def test_a_number_of_samples_that_is_none(samples):
    d = _decoder(pool_pages=40)
    before = _state(d)
    for call in (lambda: d.fork(samples), lambda: d.generate(PROMPTS, 4, 2, 2, samples=samples)):
        with pytest.raises(ValueError, match="samples"):
            call()
    _unchanged(d, before)


@pytest.mark.parametrize("prompts,samples", [([[5], [6]], 1), ([[5]], 2), ([[5, 6], [6, 7], [8, 9]], 2), ([[5], [6], [7], [8], [9]], 1), ([], 1), ([], 3)])
def test_as_many_prompts_as_the_decoder_has_requests(prompts, samples):
    # (prompts of one token go through no layer: nothing behind them would notice)
    d = _decoder(pool_pages=40)
    before = _state(d)
    with pytest.raises(ValueError, match="prompts"):
        d.generate(prompts, 4, 2, 2, samples=samples)
    _unchanged(d, before)
