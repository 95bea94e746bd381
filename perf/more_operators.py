"""What a drafting loop runs between two verify steps: products of few or many
rows with weights held in 4 bits (the draft model's projections, FFN and LM head),
the choice of the next beams from their logits, and the cache rows that follow
the chosen beams.

Weights.  A number is an E2M1 code (1 sign, 2 exponent and 1 mantissa bit: 0, 0.5,
1, 1.5, 2, 3, 4, 6 and their negatives) times a power of two that 32 consecutive
numbers of a row share: the smallest one, 2^-120 at least, with which no number of
the group exceeds 6.  A number takes the nearest code, the even one of two equally
near, and a zero the code 0.
  pack     bfloat16 weights into 4 bits, and what they then stand for
  linear   x W^T, bfloat16 or (logits) float32
  gate_up  silu(x Wg^T) * (x Wu^T)

Beams.  A group (a sample) has ``width`` beams with scores (log probabilities so
far) and logits over the vocabulary.  Candidate (beam, token) has the score
score[beam] + log softmax(logits[beam])[token]; the ``k`` best of the group are
chosen, the lower (beam, token) of equal ones first.  A beam of score -inf and a
token of logit -inf are no candidates; a beam whose last token is the end of
sequence offers that token alone, at its score.

Reorder.  Beam j of a group continues beam parents[j]: positions [begin, end) of
its cache, in all layers, become what that beam held, all beams at once.  The
parents here are such that a beam which lives on stays where it is (a second pass
then changes nothing) and ``moved`` beams of a group take another's rows.
"""

import math
from types import SimpleNamespace

import torch

own = False

# decoder shapes: hidden, query heads, KV heads, head dim, FFN, vocabulary
SHAPES = {
    "tiny": (256, 4, 2, 64, 1024, 1024),
    "1b": (2048, 32, 8, 64, 8192, 128256),
    "8b": (4096, 32, 8, 128, 14336, 128256),
    "mha": (2048, 16, 16, 128, 5632, 32000),
}


def listed():
    return [
        # a projection of a 1B decoder's weights, laid out once when the model is loaded
        dict(name="pack_1b_o", kind="pack", rows=2048, cols=2048),
        # the largest matrix of an 8B layer
        dict(name="pack_8b_gate", kind="pack", rows=14336, cols=4096),
        # one token of the last live sample through a 1B draft model: latency
        dict(name="linear_b1_1b_o", kind="linear", n=1, rows=2048, cols=2048, fp32=False),
        # 16 draft rows, the longest rows of an 8B layer
        dict(name="linear_b16_8b_down", kind="linear", n=16, rows=4096, cols=14336, fp32=False),
        # logits of three samples' eight beams
        dict(name="linear_b24_8b_head", kind="linear", n=24, rows=128256, cols=4096, fp32=True),
        # the FFN of four draft rows: two thirds of a layer's bytes
        dict(name="gate_up_b4_8b", kind="gate_up", n=4, rows=14336, cols=4096),
        # early generation, 128 samples of eight beams each: bound by the products
        dict(name="gate_up_b1024_8b", kind="gate_up", n=1024, rows=14336, cols=4096),
        # one sample's four beams over a small vocabulary: latency
        dict(name="beam_b1_w4", kind="beam", groups=1, width=4, vocab=32000, k=4, fp32=True),
        # bfloat16 logits of an odd vocabulary, more children than beams (a tree's next level)
        dict(name="beam_b17_w12_k24", kind="beam", groups=17, width=12, vocab=50001, k=24, fp32=False),
        # early generation, 128 samples of eight beams
        dict(name="beam_b128_w8", kind="beam", groups=128, width=8, vocab=128256, k=8, fp32=True),
        # eight beams of one sample, a hundred tokens into the answer
        dict(name="reorder_b1_w8", kind="reorder", pool="bf16", shape="8b", layers=16, groups=1, width=8, moved=5,
             prompt=300, tokens=100),
        # sixteen samples of eight beams over the 4-bit pool, answers of about 500 tokens
        dict(name="reorder_kv4_b16_w8", kind="reorder", pool="kv4", shape="8b", layers=8, groups=16, width=8, moved=5,
             prompt=300, tokens=500),
    ]


def draw(rng):
    def logint(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(max(a, b))))))

    def matrix():
        hidden, heads, kv, d, ffn, vocab = SHAPES[rng.choice(list(SHAPES))]
        return rng.choice([(hidden, heads * d), (kv * d, hidden), (ffn, hidden), (hidden, ffn), (vocab, hidden),
                           (logint(1, 20000), 32 * logint(1, 400)), (logint(1, 20000), 32 * logint(1, 400))])

    kind = rng.choice(["pack", "linear", "linear", "linear", "gate_up", "gate_up", "beam", "beam", "beam", "reorder",
                       "reorder"])
    if kind in ("pack", "linear", "gate_up"):
        rows, cols = matrix()
        if kind == "pack":
            most = max(1, 14336 * 4096 // cols)
            return dict(kind=kind, rows=min(rows, most), cols=cols)
        if kind == "gate_up":
            rows = min(rows, 14336)
        n = logint(1, max(1, min(1024, 1024 * 14336 * 4096 // (rows * cols))))
        if kind == "gate_up":
            return dict(kind=kind, n=n, rows=rows, cols=cols)
        return dict(kind=kind, n=n, rows=rows, cols=cols, fp32=rng.random() < 0.4)
    if kind == "beam":
        width = logint(1, 64)
        vocab = rng.choice([1024, 32000, 128256, logint(100, 130000), logint(100, 130000)])
        groups = logint(1, max(1, min(128, 128 * 8 * 128256 // (width * vocab))))
        return dict(kind=kind, groups=groups, width=width, vocab=vocab, k=logint(1, 64), fp32=rng.random() < 0.5)
    pool, width = rng.choice(["bf16", "kv4"]), logint(2, 32)
    c = dict(kind=kind, pool=pool, shape=rng.choice(["tiny", "1b", "8b", "mha"]), layers=logint(1, 16), groups=logint(1, 32),
             width=width, moved=rng.randint(1, width - 1), prompt=rng.choice([0, 1, logint(1, 500)]), tokens=logint(1, 500))
    most = 16 * 8 * 500 * 8 * 8 * 2 * 128 * (1 if pool == "kv4" else 0.27)     # numbers of the largest listed one
    while _rows(c) * _token(c) > most:
        c["tokens"] = max(1, c["tokens"] // 2)
        c["groups"] = max(1, c["groups"] // 2)
        c["prompt"] //= 2
        c["layers"] = max(1, c["layers"] // 2)
    return c


def _rows(c):
    return c["groups"] * c["width"] * (c["prompt"] + c["tokens"])


def _token(c):
    _, _, kv, d, _, _ = SHAPES[c["shape"]]
    return c["layers"] * kv * 2 * d


def work(case):
    c = SimpleNamespace(**case)
    if c.kind in ("pack", "linear", "gate_up"):
        held = c.rows * c.cols // 32 * 17
        if c.kind == "pack":          # bfloat16 in, 4 bits written and read, what they stand for out
            return {"bytes": 4 * c.rows * c.cols + 2 * held, "flops": 0}
        many = 2 if c.kind == "gate_up" else 1
        out = 4 if c.kind == "linear" and c.fp32 else 2
        return {"bytes": many * held + 2 * c.n * c.cols + out * c.n * c.rows, "flops": 2 * many * c.n * c.rows * c.cols}
    if c.kind == "beam":
        return {"bytes": c.groups * (c.width * (c.vocab * (4 if c.fp32 else 2) + 8) + 12 * c.k),
                "flops": 4 * c.groups * c.width * c.vocab}
    _, _, kv, d, _, _ = SHAPES[c.shape]
    position = c.layers * kv * (4 * d if c.pool == "bf16" else d + d // 32 + 2)
    read = min(c.moved, c.width - c.moved)        # beams that are another's parent
    return {"bytes": c.groups * c.tokens * position * (read + c.moved), "flops": 0}


# ---------------------------------------------------------------------------
# values (from the seed)
# ---------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 1_000_003 + 29)


def _normal(gen, *shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=gen)


def _weight(gen, rows, cols):
    """A trained matrix: input channels of different sizes, some of them large."""
    gain = torch.exp(0.4 * _normal(gen, cols))
    w = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    for at in range(0, rows, 8192):
        w[at:at + 8192] = (_normal(gen, min(rows, at + 8192) - at, cols, std=0.02) * gain).to(torch.bfloat16)
    return w


def _inputs(case, seed):
    """Everything that both sides and exact() start from."""
    c = SimpleNamespace(**case)
    gen = _generator(seed)
    if c.kind in ("pack", "linear", "gate_up"):
        c.weights = [_weight(gen, c.rows, c.cols) for _ in range(2 if c.kind == "gate_up" else 1)]
        if c.kind != "pack":          # normed states: some channels larger than the others
            c.x = (_normal(gen, c.n, c.cols) * torch.exp(0.5 * _normal(gen, c.cols))).to(torch.bfloat16)
        return c
    if c.kind == "beam":
        # a few likely tokens over many unlikely ones; some tokens are masked, as by a grammar
        z = _normal(gen, c.groups * c.width, c.vocab, std=2.0)
        z += 6.0 * (torch.empty_like(z).uniform_(0, 1, generator=gen) < 8.0 / c.vocab)
        z[:, torch.randint(c.vocab, (c.vocab // 50,), generator=gen, device="cuda")] = -math.inf
        c.logits = z.view(c.groups, c.width, c.vocab) if c.fp32 else z.to(torch.bfloat16).view(c.groups, c.width, c.vocab)
        c.scores = -torch.empty(c.groups, c.width, device="cuda").uniform_(0.0, 12.0, generator=gen)
        dead = torch.empty(c.groups, c.width, device="cuda").uniform_(0, 1, generator=gen)
        c.scores[dead < 0.03] = -math.inf
        c.last = torch.randint(c.vocab, (c.groups, c.width), generator=gen, device="cuda").to(torch.int32)
        c.eos = c.vocab - 1
        c.last[dead > 0.95] = c.eos
        return c
    hidden, heads, kv, d, ffn, vocab = SHAPES[c.shape]
    c.cfg = SimpleNamespace(n_layers=c.layers, hidden=hidden, n_heads=heads, n_kv_heads=kv, head_dim=d, ffn=ffn,
                            vocab=vocab, rope_theta=1e4, rms_eps=1e-5)
    # a group's beams: the survivors keep their rows, the others take a survivor's
    order = torch.argsort(torch.empty(c.groups, c.width, device="cuda").uniform_(0, 1, generator=gen), 1)
    kept = c.width - c.moved
    c.parents = torch.empty(c.groups, c.width, dtype=torch.int32, device="cuda")
    source = order[:, torch.arange(c.width, device="cuda") % kept]
    c.parents.scatter_(1, order, source.to(torch.int32))
    c.beams = c.groups * c.width
    c.end = c.prompt + c.tokens
    if c.pool == "bf16":
        c.cap = c.end + 17
        c.bytes = c.beams * c.layers * 2 * kv * c.cap * d * 2
        c.held = torch.empty(c.bytes // 2, dtype=torch.bfloat16, device="cuda")
        c.held.normal_(0.0, 1.28, generator=gen)
        c.held = c.held.view(torch.uint8)
    else:
        c.per = (c.end + 63) // 64                     # pages of a beam, all its own
        c.head_bytes = 64 * (d + d // 32 + 2)
        c.bytes = c.beams * c.per * c.layers * kv * c.head_bytes
        c.held = torch.randint(-(1 << 62), 1 << 62, (c.bytes // 8,), generator=gen, device="cuda").view(torch.uint8)
        c.pages = torch.randperm(c.beams * c.per, generator=gen, device="cuda").view(c.beams, c.per)
    return c


def _power(e):
    """2^e as double, e a whole number from -1022 to 1023."""
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def _codes(w):
    """Exponents [rows, cols / 32] and codes [rows, cols] (uint8) of a matrix."""
    y = w.double().view(w.shape[0], -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    frac, e = torch.frexp(top / 6)                     # top / 6 = frac 2^e, frac in [0.5, 1)
    e = torch.where(top > 0, e - (frac == 0.5).to(e.dtype), torch.full_like(e, -120)).clamp(-120, 127)
    e = e + (top > 6 * _power(e)).to(e.dtype)
    x = y.abs() * _power(-e)
    code = ((x > 0.25).to(torch.uint8) + (x >= 0.75) + (x > 1.25) + (x >= 1.75) + (x > 2.5)
            + (x >= 3.5) + (x > 5))
    code = code + 8 * ((y < 0) & (code > 0)).to(torch.uint8)
    return e[..., 0].to(torch.int8), code.view(w.shape)


def _pairs(code):
    """Two codes to a byte."""
    return code[:, ::2] | code[:, 1::2] << 4


def _numbers(e, pairs):
    """What exponents and pairs of codes stand for, float32 [rows, cols]."""
    code = torch.stack((pairs & 15, pairs >> 4), -1).view(pairs.shape[0], -1, 32)
    x, m = code >> 1 & 3, 0.5 * (code & 1).float()
    y = torch.where(x > 0, (1 + m) * torch.exp2(x.float() - 1), m)
    y = torch.where(code > 7, -y, y) * torch.exp2(e.float())[..., None]
    return y.view(pairs.shape[0], -1)


def _held(w):
    """A matrix in 4 bits, quantised in pieces of rows."""
    parts = [_codes(x) for x in w.split(4096)]
    return torch.cat([e for e, _ in parts]), torch.cat([_pairs(x) for _, x in parts])


def prepare(case, seed):
    s = _inputs(case, seed)
    if s.kind in ("pack", "linear", "gate_up"):
        if s.kind == "pack":
            s.w = s.weights[0]
            s.out = torch.empty_like(s.w)
        else:
            s.out = torch.empty(s.n, s.rows, device="cuda",
                                dtype=torch.float32 if s.kind == "linear" and s.fp32 else torch.bfloat16)
            if own:
                import paper_2512_04752_amd as sv
                s.m = [sv.W4Matrix(w) for w in s.weights]
            else:
                s.m = [_held(w) for w in s.weights]
        if own:
            import paper_2512_04752_amd as sv
            nbytes = sv.spec_w4_workspace_bytes(s.rows, s.cols, 1 if s.kind == "pack" else s.n)
            s.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
            if s.kind == "pack":
                s.data = torch.empty(sv.spec_w4_bytes(s.rows, s.cols), dtype=torch.uint8, device="cuda")
        del s.weights
        return s
    if s.kind == "beam":
        s.parents, s.tokens = (torch.empty(s.groups, s.k, dtype=torch.int32, device="cuda") for _ in range(2))
        s.new_scores = torch.empty(s.groups, s.k, device="cuda")
        if own:
            import paper_2512_04752_amd as sv
            nbytes = sv.spec_beam_workspace_bytes(s.groups, s.width, s.vocab, s.k)
            s.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        return s
    if own:
        import paper_2512_04752_amd as sv
        if s.pool == "bf16":
            s.kv = sv.KVPool(s.cfg, [s.cap] * s.beams)
        else:
            s.kv = sv.KV4Pool(s.cfg, s.beams, s.beams * s.per)
            for b, pages in enumerate(s.pages.tolist()):
                s.kv.map(b, pages)
        s.kv.buf[:s.bytes] = s.held
        s.held = s.kv.buf[:s.bytes]
        s.ids = torch.arange(s.beams).view(s.groups, s.width).numpy()
        s.begins, s.ends = [s.prompt] * s.groups, [s.end] * s.groups
    return s


# ---------------------------------------------------------------------------
# the pass
# ---------------------------------------------------------------------------

def _pack(s):
    e, pairs = _held(s.w)
    return {"w": _numbers(e, pairs).to(torch.bfloat16)}


def _linear(s):
    return {"out": (s.x.float() @ _numbers(*s.m[0]).T).to(s.out.dtype)}


def _gate_up(s):
    x = s.x.float()
    gate, up = x @ _numbers(*s.m[0]).T, x @ _numbers(*s.m[1]).T
    return {"out": (gate / (1 + torch.exp(-gate)) * up).to(torch.bfloat16)}


def _best(key, k):
    """The k best of each row of keys, best first, the lower index of equal ones first: (keys, indexes);
    where there are fewer than k above -inf, -inf and -1."""
    least = min(k, key.shape[1])
    last = torch.topk(key, least, 1)[0][:, -1:]
    above, at = key > last, key == last
    room = least - above.sum(1, keepdim=True)
    take = above | (at & (torch.cumsum(at, 1, dtype=torch.int32) <= room))
    index = torch.nonzero(take)[:, 1].view(-1, least)      # ascending: a stable sort keeps the lower one first
    got, order = torch.sort(torch.gather(key, 1, index), dim=1, descending=True, stable=True)
    index = torch.where(got > -math.inf, torch.gather(index, 1, order), -1)
    fill = (0, k - least)
    return torch.nn.functional.pad(got, fill, value=-math.inf), torch.nn.functional.pad(index, fill, value=-1)


def _beam(s):
    z = s.logits.double()                                  # sums of 128K terms, and candidates next to each other
    top = z.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(-1, keepdim=True))
    key = s.scores.double()[..., None] + (z - lse)
    token = torch.arange(s.vocab, device="cuda")
    ended = torch.where(token == s.eos, s.scores.double()[..., None], -math.inf)
    key = torch.where((s.last == s.eos)[..., None], ended, key)
    got, index = _best(key.view(s.groups, -1), s.k)
    parent = torch.div(index, s.vocab, rounding_mode="floor")
    token = torch.where(index < 0, -1, index - parent * s.vocab)
    return {"parents": parent.to(torch.int32), "tokens": token.to(torch.int32), "scores": got.float()}


def _reorder(s):
    kv, d, width = s.cfg.n_kv_heads, s.cfg.head_dim, s.width
    first = torch.arange(s.groups, device="cuda")[:, None] * width
    source = (first + s.parents).view(-1).long()
    if s.pool == "bf16":
        rows = s.held.view(torch.bfloat16).view(s.beams, s.layers, 2, kv, s.cap, d)[..., s.prompt:s.end, :]
        rows.copy_(rows[source])
        return {"held": s.held.view(torch.bfloat16)}
    # position by position: the low or high half of a byte of the value codes belongs to one position
    first, last = s.prompt // 64, (s.end + 63) // 64
    page = s.pages[:, first:last]
    x = s.held.view(-1, s.layers, kv, s.head_bytes)[page]  # [beams, pages, layers, heads, bytes]
    pos = torch.arange(first * 64, last * 64, device="cuda").view(-1, 64)
    inside = (pos >= s.prompt) & (pos < s.end)             # [pages, 64]
    half = 32 * d
    bits = torch.where(inside, 255, 0).to(torch.uint8)
    keys = bits.view(-1, 2, 1, 32, 1).expand(-1, -1, d // 32, -1, 16).reshape(-1, half)
    pairs = (bits.view(-1, 8, 1, 4, 2) & torch.tensor([15, 240], dtype=torch.uint8, device="cuda")).sum(-1).to(torch.uint8)
    values = pairs.expand(-1, -1, d, -1).reshape(-1, half)
    scales = [bits.repeat_interleave(n, 1) for n in (d // 32, 2)]
    mask = torch.cat((keys, values, *scales), 1)[:, None, None]
    s.held.view(-1, s.layers, kv, s.head_bytes)[page] = (x & ~mask) | (x[source] & mask)
    return {"held": s.held}


def run(state):
    s = state
    if not own:
        return {"pack": _pack, "linear": _linear, "gate_up": _gate_up, "beam": _beam, "reorder": _reorder}[s.kind](s)
    import paper_2512_04752_amd as sv
    if s.kind == "pack":
        sv.spec_w4_pack(s.w, s.data)
        sv.spec_w4_unpack(s.data, s.out)
        return {"w": s.out}
    if s.kind == "linear":
        sv.spec_w4_linear(s.m[0], s.x, s.out, workspace=s.workspace)
        return {"out": s.out}
    if s.kind == "gate_up":
        sv.spec_w4_gate_up(s.m[0], s.m[1], s.x, s.out, workspace=s.workspace)
        return {"out": s.out}
    if s.kind == "beam":
        sv.spec_beam_select(s.logits, s.scores, s.parents, s.tokens, s.new_scores, last_tokens=s.last, eos_token=s.eos,
                            workspace=s.workspace)
        return {"parents": s.parents, "tokens": s.tokens, "scores": s.new_scores}
    if s.pool == "bf16":
        sv.spec_kv_reorder(s.kv, s.ids, s.begins, s.ends, s.parents)
        return {"held": s.held.view(torch.bfloat16)}
    sv.spec_kv4_reorder(s.kv, s.ids, s.begins, s.ends, s.parents)
    return {"held": s.held}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest(w):
    """A piece of a matrix as 4 bits stand for it (doubles): every exponent from the bottom is tried."""
    y = w.to(torch.float64).reshape(-1, 32)
    grid = torch.tensor(E2M1, dtype=torch.float64, device=y.device)
    power = torch.full_like(y[:, :1], 2.0 ** -120)
    top = y.abs().amax(-1, keepdim=True)
    for e in range(-119, 128):
        power = torch.where(top > 6 * power, torch.full_like(power, 2.0 ** e), power)
        if not bool((top > 6 * power).any()):
            break
    x = y.abs() / power
    hi = torch.searchsorted(grid, x).clamp(max=7)          # the first code >= x
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - x, x - grid[lo]
    take = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (torch.sign(y) * grid[take] * power).reshape(w.shape)


def exact(case, seed):
    s = _inputs(case, seed)
    f64 = torch.float64
    if s.kind in ("pack", "linear", "gate_up"):
        pieces = [[_nearest(p) for p in w.split(8192)] if s.kind == "pack" else
                  [s.x.to(f64) @ _nearest(p).T.contiguous() for p in w.split(8192)] for w in s.weights]
        if s.kind == "pack":
            return {"w": torch.cat(pieces[0])}
        outs = [torch.cat(p, 1) for p in pieces]
        return {"out": outs[0] if s.kind == "linear" else outs[0] * torch.sigmoid(outs[0]) * outs[1]}
    if s.kind == "beam":
        parents, tokens, scores = [], [], []
        for g in range(s.groups):
            key = s.scores[g].to(f64)[:, None] + torch.log_softmax(s.logits[g].to(f64), -1)
            for w in (s.last[g] == s.eos).nonzero()[:, 0].tolist():
                key[w] = -math.inf
                key[w, s.eos] = s.scores[g, w].to(f64)
            got, at = torch.sort(key.reshape(-1), descending=True, stable=True)
            got, at = got[:s.k], at[:s.k]
            n = int((got > -math.inf).sum())
            none = [-1] * (s.k - n)
            at = at[:n].tolist()
            parents.append([i // s.vocab for i in at] + none)
            tokens.append([i % s.vocab for i in at] + none)
            scores.append(got[:n].tolist() + [-math.inf] * (s.k - n))
        return {"parents": torch.tensor(parents, dtype=torch.int32), "tokens": torch.tensor(tokens, dtype=torch.int32),
                "scores": torch.tensor(scores, dtype=f64)}
    # the cache: every beam's range from a copy of what all held before
    kv, d = s.cfg.n_kv_heads, s.cfg.head_dim
    parents = s.parents.tolist()
    old, new = s.held, s.held.clone()
    for g in range(s.groups):
        for j in range(s.width):
            src, dst = g * s.width + parents[g][j], g * s.width + j
            if src == dst:
                continue
            if s.pool == "bf16":
                a, b = (x.view(s.beams, s.layers * 2 * kv, s.cap, 2 * d) for x in (new, old))
                a[dst, :, s.prompt:s.end] = b[src, :, s.prompt:s.end]
                continue
            for p in range(s.prompt // 64, s.per):
                a = new.view(-1, s.layers * kv, s.head_bytes)[int(s.pages[dst, p])]
                b = old.view(-1, s.layers * kv, s.head_bytes)[int(s.pages[src, p])]
                lo, hi = max(0, s.prompt - 64 * p), min(64, s.end - 64 * p)
                if lo == 0 and hi == 64:
                    a.copy_(b)
                    continue
                t = torch.arange(lo, hi, device="cuda")
                for at, n in ((64 * d, d // 32), (64 * (d + d // 32), 2)):          # scales
                    a[:, at + lo * n:at + hi * n] = b[:, at + lo * n:at + hi * n]
                for c in range(d // 32):                                            # key codes
                    i = (t // 32 * 16 * d + c * 512 + t % 32 * 16)[:, None] + torch.arange(16, device="cuda")
                    a[:, i] = b[:, i]
                for x in range(lo, hi):                                             # value codes
                    i = 32 * d + x // 8 * 4 * d + torch.arange(d, device="cuda") * 4 + x % 8 // 2
                    m = 15 << 4 * (x % 2)
                    a[:, i] = (a[:, i] & (255 - m)) | (b[:, i] & m)
    return {"held": new.view(torch.bfloat16) if s.pool == "bf16" else new}
