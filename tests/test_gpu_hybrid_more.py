"""The hybrid decoder with keys and values in 8 bits and with positions of several axes: norm, append, attention and pages together, eager and captured."""
import pytest
import torch

from paper_2502_18394_amd import hybrid

pytestmark = pytest.mark.gpu
SIZES = dict(H=4, Hkv=2, layers=4, window=1024, page=16)
MODES = [dict(cache=torch.float8_e4m3fn), dict(grid=6), dict(cache=torch.float8_e4m3fn, grid=5)]


def _inputs(tokens, new, samples):
    g = torch.Generator(device="cuda").manual_seed(1)
    return torch.randint(0, 512, (tokens,), generator=g, device="cuda"), torch.rand((new, samples, 512), generator=g, device="cuda")


def _contents(m):
    return [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in (m.pool.book, m.pool.k_pages, m.pool.v_pages, m.pool.scales) if t is not None]


@pytest.mark.parametrize("mode", MODES)
def test_captured_steps_are_the_eager_ones(mode):
    prompt, noise = _inputs(90, 20, 2)
    a, ma = hybrid.run(prompt, 40, 2, 20, noise, captured=True, **SIZES, **mode)
    b, mb = hybrid.run(prompt, 40, 2, 20, noise, captured=False, **SIZES, **mode)
    assert torch.equal(a, b) and all(torch.equal(x, y) for x, y in zip(_contents(ma), _contents(mb)))
    same = noise[:, :1].expand(-1, 2, -1)
    alike, m = hybrid.run(prompt, 40, 2, 20, same, **SIZES, **mode)
    assert torch.equal(alike[0], alike[1]) and torch.equal(alike[0], a[0])
    m.release(1)
    assert int(m.pool.status[0]) == 0 and m.pool.lens.tolist() == [0, 110, 0]


@pytest.mark.parametrize("mode", MODES)
def test_keys_of_a_chunk_know_their_places(mode):
    """Keys of the first attention layer, whichever way the prompt is cut: equal up to the projection's rounding, and, in 8 bits, to a code's."""
    prompt, _ = _inputs(150, 1, 1)
    rows = []
    for chunk in (150, 17):
        m = hybrid.HybridDecoder(samples=1, **dict(SIZES, layers=2), **mode)
        m.spectral[0]["out"].zero_()                        # the window's mixture sees the whole chunk: without it the prompt is causal
        m.prompt(prompt, chunk)
        pages = m.pool.table[0, :10].long()
        k = m.pool.k_pages.float()[0, pages]
        if m.pool.scales is not None:
            k = k * m.pool.scales[0, pages, :, :, 0].repeat_interleave(16, 2)[:, :, None, :, None]
        rows.append(k.transpose(2, 3).flatten(3).transpose(1, 2).flatten(0, 1)[:150])
    # two roundings of bf16 (the projection's, whose sums may be in another order, and the key's), of components up to the largest; a code is off by half a step of 2^-4, twice
    # where a block grew, so two codes of nearly the same number are two steps apart at most
    step = 2 * 2.0 ** -8 + (4 * 2.0 ** -4 if "cache" in mode else 0)
    assert ((rows[0] - rows[1]).abs() <= step * rows[0].abs().max()).all()


def test_the_place_in_the_picture_matters():
    prompt, _ = _inputs(60, 1, 1)
    keys = []
    for grid in (0, 4, 5):
        m = hybrid.HybridDecoder(samples=1, **dict(SIZES, layers=2), grid=grid)
        m.prompt(prompt, 60)
        keys.append(m.pool.k_pages.clone())
    assert not torch.equal(keys[0], keys[1]) and not torch.equal(keys[1], keys[2])
    m = hybrid.HybridDecoder(samples=1, **dict(SIZES, layers=2), grid=5)
    assert m._positions(24, 3).tolist() == [[0, 1, 1], [4, 0, 0], [4, 0, 1]] and m._positions(7, 1, 2).tolist() == [[0, 0], [1, 1], [2, 2]]


def test_rows_that_are_one_row_and_no_layers_at_all():
    """Samples' rows that are one row's view, as a prompt's last row is before they part; a decoder without layers gives the tokens' own rows."""
    prompt, noise = _inputs(20, 1, 3)
    m = hybrid.HybridDecoder(samples=3, **SIZES)
    x = m.prompt(prompt, 20).expand(3, -1)
    assert torch.equal(m.choose(x, noise[0]), m.choose(x.clone(), noise[0]))
    m = hybrid.HybridDecoder(samples=3, **dict(SIZES, layers=0))
    assert torch.equal(m.prompt(prompt, 8), m.embed[prompt[-1:]])
    m.fork()
    assert torch.equal(m.step(prompt[:3]), m.embed[prompt[:3]])
