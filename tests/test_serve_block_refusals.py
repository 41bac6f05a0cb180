"""The serving example refuses what it cannot serve (no GPU needed: nothing gets as far as a kernel)."""
import pytest


@pytest.fixture(scope="module")
def sb():
    from paper_2501_16376_b200 import serve_block
    return serve_block


@pytest.mark.parametrize("kw", [dict(prompt=0), dict(prompt=-3), dict(steps=0), dict(n_seqs=0), dict(chunk=0), dict(budget=-1)])
def test_a_run_needs_tokens(sb, kw):
    from paper_2501_16376_b200 import synth
    args = dict(n_seqs=2, prompt=4, steps=2, budget=2)
    args.update(kw)
    with pytest.raises(ValueError):
        sb.run(synth.WORKLOADS["llama3-8b"], **args)


def test_more_tokens_than_the_cache_takes_are_refused_not_dropped(sb):
    block = sb.ServedBlock.__new__(sb.ServedBlock)
    block.length, block.capacity, block.budget = 30, 40, 24
    block._room(10)                                    # fits as it is
    for n in (17, 41):                                 # does not, evicted down to the budget either
        with pytest.raises(ValueError):
            block._room(n)
    assert block.length == 30                          # and nothing was evicted for it
