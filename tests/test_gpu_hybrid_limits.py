"""The hybrid decoder at the end of its window."""
import pytest
import torch

from paper_2502_18394_amd import hybrid

pytestmark = pytest.mark.gpu
SIZES = dict(H=4, Hkv=2, layers=2, window=256, page=16)


def _inputs(tokens, new, samples):
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randint(0, 512, (tokens,), generator=g, device="cuda"), torch.rand((new, samples, 512), generator=g, device="cuda")


def test_a_prompt_longer_than_the_window_is_refused():
    prompt, noise = _inputs(257, 1, 2)
    for chunk in (257, 64):
        with pytest.raises(ValueError, match="256"):
            hybrid.run(prompt, chunk, 2, 1, noise, **SIZES)


def test_a_pool_without_pages_is_noticed():
    """A caller's decoder whose pool is given away: the run ends with an error, not with tokens of overwritten pages."""
    prompt, _ = _inputs(100, 1, 2)
    m = hybrid.HybridDecoder(samples=2, **SIZES)
    m.pool.refs.fill_(1)
    m.prompt(prompt, 50)
    with pytest.raises(RuntimeError, match="status 1"):
        m.check()


def test_steps_end_with_the_window():
    prompt, noise = _inputs(252, 5, 2)
    tokens, m = hybrid.run(prompt, 100, 2, 4, noise, **SIZES)
    assert tokens.shape == (2, 4) and m.pool.lens.tolist() == [252, 256, 256] and int(m.pool.status[0]) == 0
    with pytest.raises(ValueError, match="256"):
        hybrid.run(prompt, 100, 2, 5, noise, **SIZES)
