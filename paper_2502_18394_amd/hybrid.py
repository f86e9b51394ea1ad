"""A decoder that keeps some attention layers beside its spectral ones, with random weights: how the library's calls go together.

    python -m paper_2502_18394_amd.hybrid [--tokens 1000] [--chunk 384] [--samples 4] [--new 32] [--layers 4] [--cache bf16|e4m3] [--grid 8]

Layers alternate: a spectral layer (token mixing by the Prefix-FFT cache) and an attention layer (queries and keys normalised and rotated,
keys and values in pages).  A prompt goes through in chunks, the sequence is forked into samples that share its full pages, each
sample draws its next tokens from given random numbers, with one captured graph a token for the attention layers' share of the work, and
at the end all but one sample are released and the pool is made dense.  The residual's addition and the norm behind it are one call.  With --cache e4m3 keys
and values are kept in 8 bits; with --grid the prompt is taken for pictures of so many patches a row, behind one another, whose tokens are turned by their place in time, row
and column.
"""
import argparse

import torch

from paper_2502_18394_amd import binding, synth


class HybridDecoder:
    """Weights and state of one prompt and its samples.  H query heads of d = 64 channels, Hkv key heads, `layers` layers, the odd ones attention."""

    def __init__(self, vocab=512, H=8, Hkv=2, layers=4, samples=4, window=4096, page=64, seed=synth.BASE_SEED, dtype=torch.bfloat16, cache=None, grid=0):
        self.H, self.Hkv, self.d, self.window, self.samples, self.dtype, self.grid = H, Hkv, 64, window, samples, dtype, grid
        self.width = H * self.d
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weights(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5).to(dtype)

        self.embed = (torch.randn((vocab, self.width), generator=g, device="cuda")).to(dtype)
        self.head = weights(self.width, vocab)
        self.attention = {}
        self.spectral = {}
        for layer in range(layers):
            if layer % 2:
                self.attention[layer] = dict(qkv=weights(self.width, (H + 2 * Hkv) * self.d), out=weights(self.width, self.width),
                                             wq=torch.ones(self.d, device="cuda"), wk=torch.ones(self.d, device="cuda"))
            else:
                self.spectral[layer] = dict(gate=binding.GateParams(synth.gate_params(seed + layer, H, self.d, window)), out=weights(self.width, self.width),
                                            cache=binding.PrefixCache(1, H, self.d, window))
        self.order = {layer: i for i, layer in enumerate(self.attention)}          # layer of the pool
        most = -(-window // page)
        self.pool = binding.KvPages.empty(max(1, len(self.order)), most * (samples + 1), Hkv, self.d, page, samples + 1, most, cache or dtype)
        # pictures: the slower half of the pairs goes by time, the others by row and column in turn
        axes = None if not grid else [0 if i >= self.d // 4 else 1 + i % 2 for i in range(self.d // 2)]
        self.rope = binding.Rope.of(self.d, 500000.0, axes=axes)
        self.all = torch.arange(samples + 1, dtype=torch.int32, device="cuda")
        self.one = torch.ones(samples + 1, dtype=torch.int32, device="cuda")
        self.tokens = 0

    def _norm(self, x, more=None):
        """(x + more, its norm): `more` is what the layer before adds to the residual."""
        if self.width * x.element_size() > binding.NORM_MOST_BYTES:
            x = self._sum(x, more)
            return x, torch.nn.functional.rms_norm(x.float(), (self.width,)).to(self.dtype)
        return binding.add_norm(x, None, more, torch.finfo(torch.float32).eps)

    @staticmethod
    def _sum(x, more):
        return x if more is None else x + more

    def _attend(self, layer, x, more, start, seqs, max_new, positions=None):
        """Attention layer on new tokens x + more [T, width]: their keys and values go into the pages, then they attend over them.  Returns (x + more, what it adds)."""
        w, T = self.attention[layer], x.shape[0]
        x, rows = self._norm(x, more)
        rows = (rows @ w["qkv"]).view(T, self.H + 2 * self.Hkv, self.d)
        q, k, v = rows.split((self.H, self.Hkv, self.Hkv), 1)                      # views: the calls take rows of any stride
        q = self.pool.append(self.order[layer], q, k, v, start, seqs, self.rope, w["wq"], w["wk"], positions=positions)
        o = self.pool.attend(self.order[layer], q, start, seqs, max_new, self.window)
        return x, o.view(T, self.width) @ w["out"]

    def _positions(self, first, count, samples=1):
        """Positions of `count` tokens from place `first` on, the same for every sample: int32 [3, samples * count], or None where the place in the sequence is the position."""
        if not self.grid:
            return None
        at = torch.arange(first, first + count, device="cuda", dtype=torch.int32)
        time, place = at // self.grid ** 2, at % self.grid ** 2
        return torch.stack((time, place // self.grid, place % self.grid)).repeat_interleave(samples, 1)

    def _room(self, more):
        """The spectral layers' window and the rows of the pool's table end here."""
        if self.tokens + more > self.window:
            raise ValueError(f"{self.tokens} tokens and {more} more: the window has {self.window}")

    def check(self):
        """What the calls on the pool found wrong (the host waits for them here, once a run; after a failed reserve they have written nothing)."""
        status = int(self.pool.status[0])
        if status:
            raise RuntimeError(f"pool status {status}")

    def prompt(self, tokens, chunk):
        """The prompt (sequence 0) in chunks; returns the last token's row."""
        self._room(tokens.numel())
        seq = self.all[:1]
        for part in tokens.split(chunk):
            T = part.numel()
            x, more = self.embed[part], None
            positions = self._positions(self.tokens, T)
            start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
            self.pool.reserve(seq, start[1:])
            for layer in range(len(self.attention) + len(self.spectral)):
                if layer in self.attention:
                    x, more = self._attend(layer, x, more, start, seq, T, positions)
                    continue
                w = self.spectral[layer]
                x, rows = self._norm(x, more)
                rows = rows.view(1, T, self.H, self.d)
                cache = w["cache"]
                cache.update(rows, rows)
                gate = binding.gate(cache.sum_q, w["gate"], 1.0 / self.window, pooled=True, phase_pos=cache.t)
                mixed = cache.readout(gate, binding.READ_WINDOW, self.dtype)[:, -T:]
                more = mixed.reshape(T, self.width) @ w["out"]
            self.tokens += T
        return self._sum(x[-1:], None if more is None else more[-1:])

    def fork(self):
        """Samples 1 .. n take over the prompt: pages shared, the last one copied; the spectral state for each of them."""
        n = self.samples
        self.pool.fork(torch.zeros(n, dtype=torch.int32, device="cuda"), self.all[1:])
        for w in self.spectral.values():
            one, many = w["cache"], binding.PrefixCache(n, self.H, self.d, self.window)
            for name in ("prefix_fft", "v_buf", "q_buf", "sum_q"):
                getattr(many, name).copy_(getattr(one, name).expand(n, *getattr(one, name).shape[1:]))
            many.c.t = one.c.t
            w["cache"] = many
        self.start = self.all.clone()                                                # one new token each: token i is sample i + 1's
        self.steps = {}

    def _captured(self, layer, x, more, positions):
        """The attention layer's step on the samples' rows, captured the first time and replayed from then on."""
        if layer not in self.steps:
            rows = [None if t is None else t.clone() for t in (x, more, positions)]
            pool = [t for t in (self.pool.book, self.pool.k_pages, self.pool.v_pages, self.pool.scales) if t is not None]
            state = [t.clone() for t in pool]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):                                          # libraries and workspaces set themselves up outside the capture
                self._attend(layer, *rows[:2], self.start, self.all[1:], 1, rows[2])
                for a, b in zip(pool, state):
                    a.copy_(b)
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = self._attend(layer, *rows[:2], self.start, self.all[1:], 1, rows[2])
            self.steps[layer] = graph, rows, out
        graph, rows, out = self.steps[layer]
        for a, b in zip(rows, (x, more, positions)):
            if a is not None:
                a.copy_(b)
        graph.replay()
        return out

    def step(self, tokens, captured=True):
        """One token for every sample; returns their rows."""
        self._room(1)
        x, more = self.embed[tokens], None
        positions = self._positions(self.tokens, 1, self.samples)
        self.pool.reserve(self.all[1:], self.one[1:])
        for layer in range(len(self.attention) + len(self.spectral)):
            if layer in self.attention:
                x, more = self._captured(layer, x, more, positions) if captured else self._attend(layer, x, more, self.start, self.all[1:], 1, positions)
            else:
                w = self.spectral[layer]
                x, rows = self._norm(x, more)
                rows = rows.view(self.samples, 1, self.H, self.d)
                more = w["cache"].step(rows, rows, w["gate"]).view(self.samples, self.width) @ w["out"]
        self.tokens += 1
        return self._sum(x, more)

    def choose(self, x, noise):
        """A token for each row, drawn with the given uniform random numbers (Gumbel's trick)."""
        logits = (self._norm(x.contiguous())[1] @ self.head).float()
        return (logits - (-noise.clamp(1e-20, 1.0).log()).log()).argmax(-1)

    def release(self, keep):
        """All but sample `keep` end, as does the prompt they were forked from; the pool becomes dense."""
        self.pool.free(torch.cat((self.all[:keep], self.all[keep + 1:])))
        self.pool.compact()


def run(prompt, chunk, samples, new, noise, captured=True, **sizes):
    """Tokens [samples, new] drawn after the prompt with noise [new, samples, vocab], and the decoder."""
    m = HybridDecoder(samples=samples, **sizes)
    x = m.prompt(prompt, chunk)
    m.fork()
    x, got = x.expand(samples, -1), []
    for i in range(new):
        got.append(m.choose(x, noise[i]))
        x = m.step(got[-1], captured)
    m.check()
    return torch.stack(got, 1), m


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 1000), ("chunk", 384), ("samples", 4), ("new", 32), ("layers", 4), ("seed", synth.BASE_SEED)):
        a.add_argument(f"--{name}", type=int, default=value)
    a.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16", help="type of the cached keys and values")
    a.add_argument("--grid", type=int, default=0, help="patches a row of the pictures that the prompt is taken for (0: a text)")
    a = a.parse_args()
    g = torch.Generator(device="cuda").manual_seed(a.seed)
    prompt = torch.randint(0, 512, (a.tokens,), generator=g, device="cuda")
    noise = torch.rand((a.new, a.samples, 512), generator=g, device="cuda")
    tokens, m = run(prompt, a.chunk, a.samples, a.new, noise, layers=a.layers, cache=torch.float8_e4m3fn if a.cache == "e4m3" else None, grid=a.grid)
    for i, row in enumerate(tokens.tolist()):
        print(f"sample {i}: {row}")
    used = int((m.pool.refs > 0).sum())
    shared = int((m.pool.refs > 1).sum())
    m.release(1)
    print(f"{m.tokens} tokens a sample; {used} pages in use, {shared} of them shared; {int(m.pool.status[2])} after the release, status {int(m.pool.status[0])}")


if __name__ == "__main__":
    main()
