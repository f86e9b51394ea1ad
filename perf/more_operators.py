"""Attention layers with a cache in 8 bits, positions of several axes and one pass for residual and norm: what these operators are measured on.

  append8   norm and rotation of the new tokens' heads, keys and values straight into pages of 8 bits
  attend8   attention of each sequence's new tokens over such pages, from one token a sequence to chunks of a document
  axes      norm and rotation where a token has a position on each of several axes (time, height, width): training, forward and
            backward ("train"), and into bfloat16 pages ("append")
  norm      a residual's addition and the norm of the sum in one pass: serving ("rows"), training, forward and backward ("train"), and with an
            output in 8 bits and a scale for each 128 channels ("coded")

Pages of 8 bits hold e4m3 numbers (four bits of exponent, three of mantissa, up to 448) in 16-byte groups, for `page` tokens of one key/value head: keys
[d / 16][page][16], a group holding adjacent channels of one token, values [page / 16][d][16], a group holding one channel of adjacent
tokens.  Each 16 tokens of a head have two scales, of keys and of values, powers of two: the smallest with which the largest magnitude is no more than 448.
Tokens that join others in such a block keep the larger of its scale and their own; where that grows, what is there is coded again.
A pool's bookkeeping is one int32 array: 8 words of status, the length of each sequence, the number of sequences that use each page, and each
sequence's row of page numbers (-1: none).
"""
import math
import random

import torch

own = False

THETA, EPS, STATUS = 500000.0, 1e-6, 8
BLOCK, LARGEST, LEAST = 16, 448.0, 2.0 ** -100            # tokens that share a scale; the largest e4m3 number; the smallest scale of pages
CODED = 128                                              # channels that share a scale of a coded norm


def listed():
    return [
        # one user's next token: the smallest call, a launch and its latency
        dict(name="append8_one", kind="append8", B=1, new=1, cached=1000, ragged=0, H=32, Hkv=8, d=64, page=64),
        # the chat turns of a batch, each of its own length
        dict(name="append8_turns", kind="append8", B=19, new=900, cached=3000, ragged=5, H=16, Hkv=4, d=128, page=32),
        # generation for one user at an ordinary context length
        dict(name="attend8_one", kind="attend8", B=1, new=1, cached=8191, ragged=0, H=32, Hkv=8, d=64, page=64, window=0),
        # generation for a batch of sequences of every length up to the longest
        dict(name="attend8_batch", kind="attend8", B=32, new=1, cached=32767, ragged=7, H=32, Hkv=8, d=64, page=64, window=0),
        # a few drafted tokens for each sequence checked at once, a sliding window, wide heads, many to a key head
        dict(name="attend8_verify", kind="attend8", B=16, new=5, cached=9000, ragged=3, H=16, Hkv=2, d=128, page=32, window=4096),
        # one chunk of a long document over what is there of it
        dict(name="attend8_chunk", kind="attend8", B=1, new=2048, cached=28672, ragged=0, H=32, Hkv=8, d=64, page=128, window=0),
        # chunks and single tokens of a batch together, small pages
        dict(name="attend8_mixed", kind="attend8", B=13, new=397, cached=5003, ragged=11, H=12, Hkv=4, d=64, page=16, window=0),
        # a training step's frames of video, forward and backward
        dict(name="axes_train", kind="axes", step="train", B=4, new=6000, H=32, Hkv=8, d=64, rot=64, axes=3, interleaved=False, io="bf16"),
        # images of a batch of conversations
        dict(name="axes_append", kind="axes", step="append", B=6, new=1021, H=16, Hkv=4, d=128, rot=128, axes=3, interleaved=True, io="bf16"),
        # one token's row between two layers
        dict(name="norm_one", kind="norm", step="rows", T=1, D=2048, io="bf16"),
        # a training step's rows, forward and backward
        dict(name="norm_train", kind="norm", step="train", T=16384, D=2048, io="bf16"),
        # a long prompt's rows for a product in 8 bits
        dict(name="norm_coded", kind="norm", step="coded", T=12001, D=4096, io="bf16"),
    ]


MOST_SCORES = 32 * 2048 * 30720         # scores of the largest listed chunk, which the plain form keeps in memory


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def draw(rng):
    kind = rng.choice(["append8", "append8", "attend8", "attend8", "attend8", "axes", "axes", "norm", "norm"])
    heads = dict(Hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 64, 128]))
    heads["H"] = heads["Hkv"] * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if g * heads["Hkv"] <= 32])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "norm":
        io = rng.choice(["bf16", "bf16", "f32"])
        step = rng.choice(["rows", "train", "coded"])
        D = CODED * _log(rng, 1, 64) if step == "coded" else 8 * _log(rng, 2, 1024)
        return dict(kind=kind, step=step, T=min(_log(rng, 1, 20000), (1 << 25) // D), D=D, io=io)
    if kind == "axes":
        case = dict(kind=kind, step=rng.choice(["train", "append"]), B=_log(rng, 1, 8), new=_log(rng, 1, 1500), rot=rng.choice([heads["d"], heads["d"], 32]),
                    axes=rng.choice([2, 3, 3, 4]), interleaved=rng.random() < 0.4, io=rng.choice(["bf16", "bf16", "f32"]), **heads)
        return case
    if kind == "append8":
        return dict(kind=kind, B=_log(rng, 1, 40), new=_log(rng, 1, 900), cached=_log(rng, 1, 3000), ragged=rng.randrange(1, 1000), page=page, **heads)
    while True:
        B, new, cached = _log(rng, 1, 48), rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 2, 2500)]), _log(rng, 1, 33000)
        if B * heads["H"] * new * (cached + new) <= MOST_SCORES // 2 and B * (cached + new) * heads["Hkv"] * heads["d"] <= 1 << 28:
            return dict(kind=kind, B=B, new=new, cached=cached, ragged=rng.choice([0, rng.randrange(1, 1000)]), page=page,
                        window=rng.choice([0, 0, 0, _log(rng, 1, 5000)]), **heads)


# ---------------------------------------------------------------- the lengths of a case, from the case alone
def _lengths(c):
    """(new tokens, tokens with them) of each sequence.  Ragged: some have one new token, one of several has none."""
    if c["kind"] == "axes":
        return [(c["new"] - 3 * b if c["new"] > 3 * b else 1, c["new"] + 7 * b + 1) for b in range(c["B"])]
    r = random.Random(c["ragged"])
    if not c["ragged"]:
        return [(c["new"], c["cached"] + c["new"])] * c["B"]
    got = []
    for b in range(c["B"]):
        n = 0 if b == 2 else 1 if r.random() < 0.4 else r.randint(1, c["new"])
        got.append((n, n + (c["cached"] if b == 0 else r.randint(0, c["cached"]))))
    return got


def _size(c):
    return 4 if c.get("io") == "f32" else 2


def work(c):
    size = _size(c)
    if c["kind"] == "norm":
        row = c["T"] * c["D"]
        if c["step"] == "train":          # both addends and both gradients read, the sum, the norm and the gradient written
            return {"bytes": 7 * row * size, "flops": 14 * row}
        out = 1 + 4 / CODED if c["step"] == "coded" else size
        return {"bytes": row * (3 * size + out), "flops": 5 * row}
    d, T = c["d"], sum(n for n, _ in _lengths(c))
    if c["kind"] == "axes":
        row = T * (c["H"] + c["Hkv"]) * d
        if c["step"] == "train":          # rows and their gradients read, both written
            return {"bytes": 4 * row * size + 4 * c["axes"] * T, "flops": 40 * row}
        return {"bytes": 2 * (row + T * c["Hkv"] * d) * size + 4 * c["axes"] * T, "flops": 12 * row}
    if c["kind"] == "append8":            # rows read, queries written, keys and values written in 8 bits with the scales of their blocks
        scales = sum((m - 1) // BLOCK - (m - n) // BLOCK + 1 for n, m in _lengths(c) if n) * 8 * c["Hkv"]
        return {"bytes": 2 * T * (2 * c["H"] + 2 * c["Hkv"]) * d + 2 * T * c["Hkv"] * d + scales, "flops": 16 * T * (c["H"] + c["Hkv"]) * d}
    keys = pairs = 0
    for n, m in _lengths(c):
        keys += (m - max(0, m - n + 1 - c["window"]) if c["window"] else m) if n else 0
        pairs += sum(min(p + 1, c["window"] or p + 1) for p in range(m - n, m))
    return {"bytes": 2 * keys * c["Hkv"] * (d + 4 / BLOCK) + 4 * T * c["H"] * d, "flops": 4 * pairs * c["H"] * d}


# ---------------------------------------------------------------- inputs
def _coded_pool(c, gen, pages):
    """Pages of 8 bits that earlier sequences have filled, their scales beside them."""
    d, page, Hkv = c["d"], c["page"], c["Hkv"]
    got = []
    for shape in ((1, pages, Hkv, d // 16, page, 16), (1, pages, Hkv, page // 16, d, 16)):
        x = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
        for i in range(0, pages, 4096):   # values around 1.2 with the scales below
            part = x[:, i:i + 4096]
            part.copy_((torch.randn(part.shape, generator=gen, device="cuda") * 90).clamp_(-LARGEST, LARGEST))
        got.append(x)
    power = torch.randint(-7, -5, (1, pages, Hkv, page // BLOCK, 2), generator=gen, device="cuda")
    return got[0], got[1], torch.exp2(power.float())


def _book(lens, table, pages):
    """The bookkeeping of sequences whose pages nobody shares."""
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[table[table >= 0].long()] = 1
    return torch.cat([torch.zeros(STATUS, dtype=torch.int32), torch.tensor(lens, dtype=torch.int32), refs, table.reshape(-1)])


def _table(lens, page, M, order):
    table, at = torch.full((len(lens), M), -1, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        m = -(-n // page)
        table[b, :m] = order[at:at + m]
        at += m
    return table


def _view(s):
    """(lengths, page numbers) in the bookkeeping."""
    book, S, P, M = s["book"], s["S"], s["P"], s["M"]
    return book[STATUS:STATUS + S], book[STATUS + S + P:].view(S, M)


def _grid(c, seed):
    """Positions [axes, T]: each sequence is a text of a few tokens, whose axes agree, and behind it a picture or frames, whose axes count apart."""
    r, parts = random.Random(seed), []
    for n, _ in _lengths(c):
        text = r.randint(0, min(n, 40))
        i, wide = torch.arange(n - text), r.randint(5, 40)
        rest = [i // wide ** 2, i // wide % wide, i % wide, i % 7][:c["axes"]] if c["axes"] > 2 else [i // wide, i % wide]
        first = r.randint(0, 90000)
        words = first + torch.arange(text).expand(c["axes"], text)
        parts.append(torch.cat((words, first + text + torch.stack(rest)), 1))
    return torch.cat(parts, 1).int()


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt, dev = torch.float32 if c.get("io") == "f32" else torch.bfloat16, "cuda"
    s = dict(case=c)

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dtype)

    if c["kind"] == "norm":
        T, D = c["T"], c["D"]
        s["x"], s["delta"], s["w"] = normal(T, D, scale=3.0), normal(T, D), 1 + normal(D, scale=0.1, dtype=torch.float32)
        if c["step"] == "train":
            s["dy"], s["dsum"] = normal(T, D), normal(T, D)
        return s
    d = c["d"]
    # weights of the norms around 0.8, as a trained model's
    s["wq"], s["wk"] = (0.8 + normal(d, scale=0.05, dtype=torch.float32) for _ in "qk")
    rot = c.get("rot", d)
    s["freq"] = (THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).to(dev)
    news, lens = zip(*_lengths(c))
    T = sum(news)
    s["T"] = T
    if c["kind"] == "axes":
        # the slower pairs go by time, the others by the other axes in turn
        n = c["axes"]
        s["axis"] = torch.tensor([0 if i >= rot // 2 - rot // 8 else (1 + i % (n - 1)) for i in range(rot // 2)], dtype=torch.int32)
        s["positions"] = _grid(c, seed).to(dev)
        s["q"] = normal(T, c["H"], d)
        kv = normal(T, 2, c["Hkv"], d)                         # keys and values as one projection leaves them
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        if c["step"] == "train":
            s["dq"], s["dk"] = normal(T, c["H"], d), normal(T, c["Hkv"], d)
            _plan(s, c)
            return s
    page = c.get("page", 64)
    M = max(1, -(-max(lens) // page))
    P = sum(-(-n // page) for n in lens) + 3
    if c["kind"] == "axes":
        E = 16 // _size(c)
        s["k_pages"], s["v_pages"] = normal(1, P, c["Hkv"], d // E, page, E), normal(1, P, c["Hkv"], page // E, d, E)
    else:
        s["k_pages"], s["v_pages"], s["scales"] = _coded_pool(c, gen, P)
        s["q"] = normal(T, c["H"], d, scale=2.0)
    # a batch's sequences are rows of the pool's table in an order of their own
    seqs = torch.randperm(c["B"], generator=host).int()
    rows = [0] * c["B"]
    for b, at in enumerate(seqs.tolist()):
        rows[at] = lens[b]
    book = _book(rows, _table(rows, page, M, torch.randperm(P, generator=host).int()), P)
    start = torch.tensor((0,) + news).cumsum(0).int()
    s.update(book=book.to(dev), S=c["B"], P=P, M=M, page=page, seqs=seqs.to(dev), start=start.to(dev), max_new=max(news), max_len=max(lens))
    if c["kind"] == "append8":
        kv = normal(T, 2, c["Hkv"], d)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
    _plan(s, c)
    return s


def _plan(s, c):
    if own:
        from paper_2502_18394_amd import binding
        s["rope"] = binding.Rope(s["freq"], interleaved=c.get("interleaved", False), axes=s.get("axis"))
        if "book" in s:
            s["pool"] = binding.KvPages(s["k_pages"], s["v_pages"], s["book"], s["S"], s["M"], scales=s.get("scales"))


# ---------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "norm":
        return _plain_norm(s, c)
    if c["kind"] == "attend8":
        return _plain_attend(s, c)
    if c["kind"] == "append8":
        return _plain_append8(s, c)
    return _plain_train(s, c) if c["step"] == "train" else _plain_append(s, c)


def _run_own(s, c):
    from paper_2502_18394_amd import binding
    if c["kind"] == "norm":
        if c["step"] == "coded":
            total, codes, scales = binding.add_norm(s["x"], s["w"], s["delta"], EPS, dtype=torch.float8_e4m3fn)
            return dict(sum=total, codes=codes, scales=scales)
        total, y = binding.add_norm(s["x"], s["w"], s["delta"], EPS)
        if c["step"] == "rows":
            return dict(sum=total, y=y)
        gx, gw = binding.add_norm_backward(s["dy"], total, s["w"], s["dsum"], EPS)
        return dict(sum=total, y=y, gx=gx, gw=gw)
    if c["kind"] == "axes" and c["step"] == "train":
        q, k = binding.qk_norm_rotate(s["q"], s["k"], s["positions"], s["rope"], s["wq"], s["wk"], EPS)
        gq, gk, gwq, gwk = binding.qk_norm_rotate_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["rope"], s["wq"], s["wk"], EPS)
        return dict(q=q, k=k, gq=gq, gk=gk, gwq=gwq, gwk=gwk)
    pool = s["pool"]
    if c["kind"] == "attend8":
        out, lse = pool.attend(0, s["q"], s["start"], s["seqs"], s["max_new"], s["max_len"], window=c["window"], want_lse=True)
        return dict(out=out, lse=lse)
    q = pool.append(0, s["q"], s["k"], s["v"], s["start"], s["seqs"], s["rope"], s["wq"], s["wk"], EPS, positions=s.get("positions"))
    if c["kind"] == "append8":
        return dict(q=q, k=s["k_pages"], v=s["v_pages"], scales=s["scales"])
    return dict(q=q, k=s["k_pages"], v=s["v_pages"])


# ---------------------------------------------------------------- plain forms
def _plain_norm(s, c):
    x, w = s["x"], s["w"]
    total = (x.float() + s["delta"].float()).to(x.dtype)
    t = total.float()
    r = torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS)
    unit = t * r
    y = unit * w
    if c["step"] == "coded":
        parts = y.view(c["T"], -1, CODED)
        scales = parts.abs().amax(-1) / LARGEST
        codes = (parts / torch.where(scales > 0, scales, 1.0)[..., None]).clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn)
        return dict(sum=total, codes=codes.view(c["T"], -1), scales=scales)
    if c["step"] == "rows":
        return dict(sum=total, y=y.to(x.dtype))
    g = s["dy"].float()
    h = g * w
    gx = r * (h - unit * (h * unit).mean(-1, keepdim=True)) + s["dsum"].float()
    gw = (g * unit).sum(0, dtype=torch.float64).float()
    return dict(sum=total, y=y.to(x.dtype), gx=gx.to(x.dtype), gw=gw)


def _turns(s, positions):
    """cos and sin [T, 1, rot / 2] of each token's angles, which are formed in 64 bits.  positions [T], or [axes, T]."""
    at = positions.double()
    at = at[:, None] if at.dim() == 1 else at[s["axis"].long().to(at.device)].T
    angle = (at * s["freq"])[:, None]
    return angle.cos().float(), angle.sin().float()


def _rotate(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _unit(x):
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_train(s, c):
    cos, sin = _turns(s, s["positions"])
    out = {}
    for n, w in (("q", s["wq"]), ("k", s["wk"])):
        x = s[n]
        unit, r = _unit(x)
        out[n] = _rotate(unit * w, cos, sin, c["interleaved"]).to(x.dtype)
        g = _rotate(s["d" + n].float(), cos, -sin, c["interleaved"])
        out["gw" + n] = (g * unit).sum((0, 1), dtype=torch.float64).float()
        h = g * w
        out["g" + n] = (r * (h - unit * (h * unit).mean(-1, keepdim=True))).to(x.dtype)
    return out


def _tokens(s):
    """(sequence's place in the batch, its row of the table, place in the sequence) of each new token."""
    lens, _ = _view(s)
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["start"][1:].long(), t, right=True)
    row = s["seqs"].long()[b]
    return b, row, lens[row].long() - s["start"][b + 1].long() + t


def _heads(s, positions, interleaved):
    cos, sin = _turns(s, positions)
    return (_rotate(_unit(s[n])[0] * s["w" + n], cos, sin, interleaved) for n in "qk")


def _plain_append(s, c):
    E, page = 16 // _size(c), s["page"]
    _, row, at = _tokens(s)
    q, k = (x.to(s["q"].dtype) for x in _heads(s, s["positions"], c["interleaved"]))
    number, slot = _view(s)[1][row, at // page].long(), at % page
    s["k_pages"][0][number, :, :, slot, :] = k.reshape(s["T"], c["Hkv"], c["d"] // E, E)
    s["v_pages"][0][number, :, slot // E, :, slot % E] = s["v"]
    return dict(q=q, k=s["k_pages"], v=s["v_pages"])


def _scale_of(amax):
    """The smallest power of two s with amax <= 448 s = 0.875 * 2^9 s, no less than 2^-100."""
    m, e = torch.frexp(amax)
    return torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875).int()).clamp(min=LEAST)


def _plain_append8(s, c):
    T, Hkv, d, page = s["T"], c["Hkv"], c["d"], s["page"]
    b, row, at = _tokens(s)
    q, k = _heads(s, at, False)
    lens, table = _view(s)
    # the blocks that get tokens, in the order of the tokens
    block = table[row, at // page].long() * (page // BLOCK) + at % page // BLOCK
    first = torch.ones_like(block, dtype=torch.bool)
    first[1:] = block[1:] != block[:-1]
    mine = first.long().cumsum(0) - 1
    block, had = block[first], (at % BLOCK)[first]            # tokens that a block holds already
    slot = at % BLOCK
    number, part = block // (page // BLOCK), block % (page // BLOCK)
    keep = (torch.arange(BLOCK, device="cuda") < had[:, None])[:, None, None, :]
    k_bytes, v_bytes = s["k_pages"][0], s["v_pages"][0]
    new = {}
    for i, x in enumerate((k, s["v"].float())):
        if i == 0:      # [blocks, Hkv, d, 16 tokens]
            old = k_bytes.view(torch.uint8).unflatten(3, (-1, BLOCK))[number, :, :, part].permute(0, 1, 2, 4, 3).reshape(-1, Hkv, d, BLOCK)
        else:
            old = v_bytes.view(torch.uint8)[number, :, part]
        was = s["scales"][0, number, :, part, i]
        amax = torch.zeros(block.numel(), Hkv, device="cuda")
        amax.scatter_reduce_(0, mine[:, None].expand(-1, Hkv), x.abs().amax(-1), "amax")
        scale = torch.maximum(_scale_of(amax), torch.where(had[:, None] > 0, was, 0.0))
        value = old.view(torch.float8_e4m3fn).float() * (was / scale)[..., None, None]
        again = value.to(torch.float8_e4m3fn).view(torch.uint8)
        coded = torch.where(keep, again, old)
        coded[mine, :, :, slot] = (x / scale[mine][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        new[i] = coded, scale
    coded, scale = new[0]
    k_bytes.view(torch.uint8).unflatten(3, (-1, BLOCK))[number, :, :, part] = coded.view(-1, Hkv, d // 16, 16, BLOCK).transpose(-1, -2)
    s["scales"][0, number, :, part, 0] = scale
    coded, scale = new[1]
    v_bytes.view(torch.uint8)[number, :, part] = coded
    s["scales"][0, number, :, part, 1] = scale
    return dict(q=q.to(s["q"].dtype), k=s["k_pages"], v=s["v_pages"], scales=s["scales"])


def _plain_attend(s, c):
    B, H, Hkv, d, page, n, m = c["B"], c["H"], c["Hkv"], c["d"], c["page"], s["max_new"], s["max_len"]
    lens, table = _view(s)
    seqs = s["seqs"].long()
    number = table[seqs, :-(-m // page)].clamp(min=0).long()                      # [B, pages]
    ks, vs = s["scales"][0][number].unbind(-1)                                   # [B, pages, Hkv, blocks]
    keys = s["k_pages"].view(torch.uint8)[0][number].view(torch.float8_e4m3fn).float()
    keys = keys.unflatten(4, (-1, BLOCK)) * ks[:, :, :, None, :, None, None]
    keys = keys.flatten(4, 5).permute(0, 2, 3, 5, 1, 4).reshape(B, Hkv, d, -1)[..., :m]
    vals = s["v_pages"].view(torch.uint8)[0][number].view(torch.float8_e4m3fn).float() * vs[..., None, None]
    vals = vals.permute(0, 2, 1, 3, 5, 4).reshape(B, Hkv, -1, d)[:, :, :m]
    b, _, at = _tokens(s)
    have, total = (s["start"][1:] - s["start"][:-1]).long(), lens[seqs].long()
    i = torch.arange(n, device="cuda")
    q = s["q"][(s["start"][:-1].long()[:, None] + i).clamp(max=s["T"] - 1)].float()   # [B, n, H, d]
    q = q.view(B, n, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    p = torch.matmul(q, keys).view(B, Hkv, H // Hkv, n, m) * (1 / math.sqrt(d))
    where = ((total - have)[:, None] + i)[:, None, None, :, None]                  # position of each query
    key = torch.arange(m, device="cuda")
    hidden = key > where
    if c["window"]:
        hidden = hidden | (key <= where - c["window"])
    p.masked_fill_(hidden, -math.inf)
    top = p.amax(-1, keepdim=True).clamp(min=-3e38)
    p.sub_(top).exp_()
    total_p = p.sum(-1, keepdim=True)
    # what lies beyond a sequence's end is another's, or nothing
    vals = vals.masked_fill((key >= total[:, None])[:, None, :, None], 0)
    o = torch.matmul(p.view(B, Hkv, -1, m), vals).view(B, Hkv, H // Hkv, n, d)
    o = torch.where(total_p > 0, o / total_p, 0).permute(0, 3, 1, 2, 4).reshape(B, n, H, d)
    lse = (top + total_p.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, H)
    local = torch.arange(s["T"], device="cuda") - s["start"].long()[b]
    return dict(out=o[b, local].to(s["q"].dtype), lse=lse[b, local])


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "norm":
        return _exact_norm(s, c)
    if c["kind"] == "attend8":
        return _exact_attend(s, c)
    if c["kind"] == "append8":
        return _exact_append8(s, c)
    return _exact_train(s, c) if c["step"] == "train" else _exact_append(s, c)


def _exact_norm(s, c):
    x, w = s["x"].double(), s["w"].double().requires_grad_()
    total = (x + s["delta"].double()).to(s["x"].dtype).double().requires_grad_()      # what is kept of the sum is the input of the norm
    y = total / (total.pow(2).sum(-1, keepdim=True) / c["D"] + EPS).sqrt() * w
    if c["step"] == "train":
        gx, gw = torch.autograd.grad(y, (total, w), s["dy"].double())
        return dict(sum=(x + s["delta"].double()), y=y.detach(), gx=gx + s["dsum"].double(), gw=gw)
    if c["step"] == "rows":
        return dict(sum=(x + s["delta"].double()), y=y.detach())
    y = y.detach().unflatten(-1, (-1, CODED))
    scales = y.abs().amax(-1) / LARGEST
    return dict(sum=(x + s["delta"].double()), codes=(y / scales.clamp(min=1e-300)[..., None]).flatten(1), scales=scales)


def _exact_heads(x, w, angle, interleaved):
    """Norm and rotation, the pairs as complex numbers."""
    y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w
    half = angle.shape[-1]
    turned, rest = y[..., :2 * half], y[..., 2 * half:]
    pair = turned.unflatten(-1, (half, 2)) if interleaved else turned.unflatten(-1, (2, half)).transpose(-1, -2)
    z = torch.view_as_complex(pair.contiguous()) * torch.polar(torch.ones_like(angle), angle)
    z = torch.view_as_real(z)
    return torch.cat((z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2), rest), -1)


def _exact_angle(s):
    at = torch.stack([s["positions"][a] for a in s["axis"].tolist()], -1)
    return (at.double() * s["freq"])[:, None]


def _exact_train(s, c):
    angle, got = _exact_angle(s), {}
    for n in "qk":
        x, w = s[n].double().requires_grad_(), s["w" + n].double().requires_grad_()
        y = _exact_heads(x, w, angle, c["interleaved"])
        got["g" + n], got["gw" + n] = torch.autograd.grad(y, (x, w), s["d" + n].double())
        got[n] = y.detach()
    return got


def _sequences(s):
    """(first new token, behind the last, row of the table, place of the first in the sequence) of the sequences that have new tokens."""
    lens, start = _view(s)[0].tolist(), s["start"].tolist()
    for b, row in enumerate(s["seqs"].tolist()):
        lo, hi = start[b], start[b + 1]
        if lo < hi:
            yield lo, hi, row, lens[row] - (hi - lo)


def _exact_append(s, c):
    E, page, table = 16 // _size(c), s["page"], _view(s)[1].tolist()
    k, v, angle = s["k_pages"].double(), s["v_pages"].double(), _exact_angle(s)
    q = _exact_heads(s["q"].double(), s["wq"].double(), angle, c["interleaved"])
    key, val = _exact_heads(s["k"].double(), s["wk"].double(), angle, c["interleaved"]), s["v"].double()
    for lo, hi, row, had in _sequences(s):
        t = lo
        while t < hi:                                  # what goes into one page
            at = had + t - lo
            n = min(hi - t, page - at % page)
            number, slots = table[row][at // page], torch.arange(at % page, at % page + n, device="cuda")
            k[0, number, :, :, slots] = key[t:t + n].unflatten(-1, (-1, E)).permute(1, 2, 0, 3)
            v[0, number, :, slots // E, :, slots % E] = val[t:t + n]
            t += n
    return dict(q=q, k=k, v=v)


def _exact_append8(s, c):
    page, table, d, Hkv = s["page"], _view(s)[1].tolist(), c["d"], c["Hkv"]
    k, v, scales = s["k_pages"].double(), s["v_pages"].double(), s["scales"].double()
    q, keys, steps = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["k"].shape, dtype=torch.float64, device="cuda"), []
    for lo, hi, row, had in _sequences(s):
        angle = (torch.arange(had, had + hi - lo, device="cuda").double()[:, None] * s["freq"])[:, None]
        q[lo:hi], keys[lo:hi] = (_exact_heads(s[n][lo:hi].double(), s["w" + n].double(), angle, False) for n in "qk")
        t = lo
        while t < hi:                                  # what goes into one block
            at = had + t - lo
            n = min(hi - t, BLOCK - at % BLOCK)
            steps.append((table[row][at // page], at % page // BLOCK, at % BLOCK, t, n))
            t += n
    if len(steps) > 6000:
        return None
    for number, part, slot, t, n in steps:
        old = k[0, number, :, :, BLOCK * part:BLOCK * part + slot].transpose(1, 2).flatten(2), v[0, number, :, part, :, :slot].transpose(1, 2)
        for i, (x, there) in enumerate(zip((keys, s["v"].double()), old)):
            x = x[t:t + n].transpose(0, 1)
            scale = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / LARGEST)).clamp(min=-100))
            was = scales[0, number, :, part, i]
            if slot:
                scale = torch.maximum(scale, was)
            whole = torch.cat(((there * (was / scale)[:, None, None]).to(torch.float8_e4m3fn).double() if slot else there, x / scale[:, None, None]), 1)
            if i == 0:
                k[0, number, :, :, BLOCK * part:BLOCK * part + slot + n] = whole.unflatten(2, (-1, 16)).transpose(1, 2)
            else:
                v[0, number, :, part, :, :slot + n] = whole.transpose(1, 2)
            scales[0, number, :, part, i] = scale
    return dict(q=q, k=k, v=v, scales=scales)


def _exact_attend(s, c):
    H, Hkv, d, table = c["H"], c["Hkv"], c["d"], _view(s)[1]
    out = torch.zeros(s["T"], H, d, dtype=torch.float64, device="cuda")
    lse = torch.full((s["T"], H), -math.inf, dtype=torch.float64, device="cuda")
    for lo, hi, row, had in _sequences(s):
        m = had + hi - lo
        numbers = table[row, :-(-m // c["page"])].long()
        for g in range(Hkv):
            scale = s["scales"][0, numbers, g].double().repeat_interleave(BLOCK, 1).flatten(0, 1)[:m, None]        # of each token: [m, 1, 2]
            key = s["k_pages"].view(torch.uint8)[0, numbers, g].view(torch.float8_e4m3fn).double().transpose(1, 2).reshape(-1, d)[:m] * scale[..., 0]
            val = s["v_pages"].view(torch.uint8)[0, numbers, g].view(torch.float8_e4m3fn).double().transpose(2, 3).reshape(-1, d)[:m] * scale[..., 1]
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                pos = torch.arange(had, m, device="cuda")[:, None]
                at = torch.arange(m, device="cuda")[None]
                seen = (at <= pos) & ((at > pos - c["window"]) if c["window"] else True)
                score = torch.where(seen, s["q"][lo:hi, h].double() @ key.T / math.sqrt(d), -math.inf)
                lse[lo:hi, h] = torch.logsumexp(score, -1)
                out[lo:hi, h] = torch.softmax(score, -1) @ val
    return dict(out=out, lse=lse)
