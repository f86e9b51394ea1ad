"""A decoder that keeps some attention layers beside its spectral ones, with random weights: how the library's calls go together.

    python -m paper_2502_18394_amd.hybrid [--tokens 1000] [--chunk 384] [--samples 4] [--new 32] [--layers 4]

Layers alternate: a spectral layer (token mixing by the Prefix-FFT cache) and an attention layer (queries and keys normalised and rotated,
keys and values in pages).  A prompt goes through in chunks, the sequence is forked into samples that share its full pages, each
sample draws its next tokens from given random numbers, with one captured graph a token for the attention layers' share of the work, and
at the end all but one sample are released and the pool is made dense.
"""
import argparse

import torch

from paper_2502_18394_amd import binding, synth


class HybridDecoder:
    """Weights and state of one prompt and its samples.  H query heads of d = 64 channels, Hkv key heads, `layers` layers, the odd ones attention."""

    def __init__(self, vocab=512, H=8, Hkv=2, layers=4, samples=4, window=4096, page=64, seed=synth.BASE_SEED, dtype=torch.bfloat16):
        self.H, self.Hkv, self.d, self.window, self.samples, self.dtype = H, Hkv, 64, window, samples, dtype
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
        self.pool = binding.KvPages.empty(max(1, len(self.order)), most * (samples + 1), Hkv, self.d, page, samples + 1, most, dtype)
        self.rope = binding.Rope.of(self.d, 500000.0)
        self.all = torch.arange(samples + 1, dtype=torch.int32, device="cuda")
        self.one = torch.ones(samples + 1, dtype=torch.int32, device="cuda")
        self.tokens = 0

    def _norm(self, x):
        return torch.nn.functional.rms_norm(x.float(), (self.width,)).to(self.dtype)

    def _attend(self, layer, x, start, seqs, max_new):
        """Attention layer on new tokens x [T, width]: their keys and values go into the pages, then they attend over them."""
        w, T = self.attention[layer], x.shape[0]
        rows = (self._norm(x) @ w["qkv"]).view(T, self.H + 2 * self.Hkv, self.d)
        q, k, v = rows.split((self.H, self.Hkv, self.Hkv), 1)                      # views: the calls take rows of any stride
        q = self.pool.append(self.order[layer], q, k, v, start, seqs, self.rope, w["wq"], w["wk"])
        o = self.pool.attend(self.order[layer], q, start, seqs, max_new, self.window)
        return x + o.view(T, self.width) @ w["out"]

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
            x = self.embed[part]
            start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
            self.pool.reserve(seq, start[1:])
            for layer in range(len(self.attention) + len(self.spectral)):
                if layer in self.attention:
                    x = self._attend(layer, x, start, seq, T)
                    continue
                w = self.spectral[layer]
                rows = self._norm(x).view(1, T, self.H, self.d)
                cache = w["cache"]
                cache.update(rows, rows)
                gate = binding.gate(cache.sum_q, w["gate"], 1.0 / self.window, pooled=True, phase_pos=cache.t)
                mixed = cache.readout(gate, binding.READ_WINDOW, self.dtype)[:, -T:]
                x = x + mixed.reshape(T, self.width) @ w["out"]
            self.tokens += T
        return x[-1:]

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

    def _captured(self, layer, x):
        """The attention layer's step on the samples' rows, captured the first time and replayed from then on."""
        if layer not in self.steps:
            rows = x.clone()
            state = [t.clone() for t in (self.pool.book, self.pool.k_pages, self.pool.v_pages)]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):                                          # libraries and workspaces set themselves up outside the capture
                self._attend(layer, rows, self.start, self.all[1:], 1)
                for a, b in zip((self.pool.book, self.pool.k_pages, self.pool.v_pages), state):
                    a.copy_(b)
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = self._attend(layer, rows, self.start, self.all[1:], 1)
            self.steps[layer] = graph, rows, out
        graph, rows, out = self.steps[layer]
        rows.copy_(x)
        graph.replay()
        return out

    def step(self, tokens, captured=True):
        """One token for every sample; returns their rows."""
        self._room(1)
        x = self.embed[tokens]
        self.pool.reserve(self.all[1:], self.one[1:])
        for layer in range(len(self.attention) + len(self.spectral)):
            if layer in self.attention:
                x = self._captured(layer, x) if captured else self._attend(layer, x, self.start, self.all[1:], 1)
            else:
                w = self.spectral[layer]
                rows = self._norm(x).view(self.samples, 1, self.H, self.d)
                x = x + w["cache"].step(rows, rows, w["gate"]).view(self.samples, self.width) @ w["out"]
        self.tokens += 1
        return x

    def choose(self, x, noise):
        """A token for each row, drawn with the given uniform random numbers (Gumbel's trick)."""
        logits = (self._norm(x) @ self.head).float()
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
    a = a.parse_args()
    g = torch.Generator(device="cuda").manual_seed(a.seed)
    prompt = torch.randint(0, 512, (a.tokens,), generator=g, device="cuda")
    noise = torch.rand((a.new, a.samples, 512), generator=g, device="cuda")
    tokens, m = run(prompt, a.chunk, a.samples, a.new, noise, layers=a.layers)
    for i, row in enumerate(tokens.tolist()):
        print(f"sample {i}: {row}")
    used = int((m.pool.refs > 0).sum())
    shared = int((m.pool.refs > 1).sum())
    m.release(1)
    print(f"{m.tokens} tokens a sample; {used} pages in use, {shared} of them shared; {int(m.pool.status[2])} after the release, status {int(m.pool.status[0])}")


if __name__ == "__main__":
    main()
