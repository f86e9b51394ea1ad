"""The decoder with attention layers beside spectral ones: chunks, forks, samples, a captured decode step, release."""
import pytest
import torch

from paper_2502_18394_amd import hybrid

pytestmark = pytest.mark.gpu
SIZES = dict(H=4, Hkv=2, layers=4, window=1024, page=16)


def _inputs(tokens, new, samples):
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randint(0, 512, (tokens,), generator=g, device="cuda"), torch.rand((new, samples, 512), generator=g, device="cuda")


def test_samples_are_their_own_and_share_the_prompt():
    prompt, noise = _inputs(203, 12, 3)
    tokens, m = hybrid.run(prompt, 64, 3, 12, noise, **SIZES)
    # sample i with sample 0's noise is sample 0; the samples' order does not matter
    same = noise[:, :1].expand(-1, 3, -1)
    alike, _ = hybrid.run(prompt, 64, 3, 12, same, **SIZES)
    assert torch.equal(alike[0], alike[1]) and torch.equal(alike[0], alike[2]) and torch.equal(alike[0], tokens[0])
    assert not torch.equal(tokens[0], tokens[1])
    turned, _ = hybrid.run(prompt, 64, 3, 12, noise[:, [2, 0, 1]], **SIZES)
    assert torch.equal(turned, tokens[[2, 0, 1]])
    # pages: 12 full ones of the prompt with four users, a last one and what came after for the prompt and each sample
    refs = m.pool.refs.tolist()
    assert m.pool.lens.tolist() == [203, 215, 215, 215] and int(m.pool.status[0]) == 0
    assert sum(r == 4 for r in refs) == 12 and sum(r == 1 for r in refs) == 1 + 3 * 2
    m.release(2)
    assert m.pool.lens.tolist() == [0, 0, 215, 0] and [r for r in m.pool.refs.tolist() if r] == [1] * 14
    assert int(m.pool.status[2]) == 14 and sorted(m.pool.table[2, :14].tolist()) == list(range(14))


def test_captured_steps_are_the_eager_ones():
    prompt, noise = _inputs(90, 20, 2)
    a, ma = hybrid.run(prompt, 90, 2, 20, noise, captured=True, **SIZES)
    b, mb = hybrid.run(prompt, 90, 2, 20, noise, captured=False, **SIZES)
    assert torch.equal(a, b) and torch.equal(ma.pool.book, mb.pool.book)
    assert torch.equal(ma.pool.k_pages, mb.pool.k_pages) and torch.equal(ma.pool.v_pages, mb.pool.v_pages)


def test_pages_after_chunks_are_those_of_one_piece():
    """Rotated keys of the first attention layer see every earlier layer's work; they agree to the rounding of bf16 rows whichever way the prompt was cut."""
    prompt, _ = _inputs(150, 1, 1)
    rows = []
    for chunk in (150, 64, 17):
        m = hybrid.HybridDecoder(samples=1, **dict(SIZES, layers=2))
        m.spectral[0]["out"].zero_()                        # the window's mixture sees the whole chunk: without it the prompt is causal
        m.prompt(prompt, chunk)
        pages = m.pool.table[0, :10].long()
        rows.append(m.pool.k_pages[0, pages].float())
        assert m.pool.lens.tolist() == [150, 0]
    # a product of other shape may add in another order: one step of a projection's rounding, one of the key's, of components of size 1 (norm) to 8
    for other in rows[1:]:
        assert ((rows[0] - other).abs() <= 2 * 2.0 ** -8 * rows[0].abs().max()).all()
