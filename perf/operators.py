"""The operators that serve requests from a paged key-value cache, as measurable cases.

Three operators over one cache layout and one batch description:
  append   new tokens' keys and values into the cache, per-head norms and rotary positions on the way;
           the rotated queries come out beside it
  decode   attention of one new token per sequence over its pages
  prompt   attention of many new tokens per sequence, causal, behind what the cache already holds;
           both with or without a sliding window and a few first tokens that stay visible

Cache: K and V fp16 [pages][key heads][tokens of a page][head width]; a page table int32 [sequences][pages],
cached tokens int32 [sequences] (the new ones counted) and, where a sequence has more than one new token, the
first row of each in the ragged token tensors, int32 [sequences + 1].

`listed()` gives the fixed cases, `draw(rng)` one more of the same ranges, `prepare(case, seed)` what a
serving program holds before a call, `run(state)` one pass, `work(case)` the bytes and operations a pass
cannot do without, `exact(case, seed)` the results in 64 bits.  With `own` false `run` computes the operators
from elementary torch operations in 32 bits, with `own` true it calls the library.
"""
import math
from types import SimpleNamespace

import torch

own = False

THETA = 10000.0
EPS = 1e-5
# (query heads, key heads, head width): the 7B, 13B, 70B and Mixtral shapes of the benchmark, the toy shapes of
# the tests, and generic ones (one key head for all, a ratio that is no power of two)
HEADS = [(32, 32, 128), (40, 40, 128), (64, 8, 128), (32, 8, 128), (8, 2, 64), (4, 4, 64), (16, 1, 128), (9, 3, 64)]


def listed():
    return [
        # one decode step of the 7B shape at the benchmark's context, one request: launch latency
        _case("append-1", "append", 1, 1, 511, (32, 32, 128), 16),
        # a full decode batch with norms of queries and keys, every request at its own length
        _case("append-64", "append", 64, 1, 4095, (32, 8, 128), 16, norm=True),
        # prompts of several requests in one call, ragged
        _case("append-prompts", "append", 7, 2039, 700, (64, 8, 128), 64),
        # attention of that single 7B-shape token
        _case("decode-1", "decode", 1, 1, 512, (32, 32, 128), 16),
        # eight requests of the 70B shape, as many as the batched layer takes
        _case("decode-8", "decode", 8, 1, 517, (64, 8, 128), 16),
        # a serving batch whose lengths spread from a few tokens to the longest
        _case("decode-64-ragged", "decode", 64, 1, 8190, (32, 8, 128), 16),
        # one long document
        _case("decode-long", "decode", 1, 1, 131070, (64, 8, 128), 64),
        # long chats under a window, the first four tokens kept
        _case("decode-window", "decode", 32, 1, 16384, (32, 8, 128), 32, window=1024, sinks=4),
        # a short question, toy shape: latency
        _case("prompt-77", "prompt", 1, 77, 0, (8, 2, 64), 16),
        # several prompts of different lengths, some behind earlier turns
        _case("prompt-ragged", "prompt", 6, 1501, 2600, (32, 8, 128), 16),
        # a long prompt from its beginning, as many key heads as query heads
        _case("prompt-8192", "prompt", 1, 8192, 0, (32, 32, 128), 64),
        # two long prompts under a window
        _case("prompt-window", "prompt", 2, 7993, 0, (32, 8, 128), 16, window=1024, sinks=4),
    ]


def _case(name, kind, seqs, new, past, heads, page, norm=False, window=0, sinks=0):
    """`new`: new tokens of the longest sequence; `past`: tokens that the longest cache holds before them."""
    c = {"kind": kind, "seqs": seqs, "new": new, "past": past, "heads": heads[0], "kv_heads": heads[1], "hd": heads[2],
         "page": page, "norm": norm, "window": window, "sinks": sinks}
    return c if name is None else {"name": name, **c}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "decode", "prompt"])
        heads, page = rng.choice(HEADS), rng.choice([16, 32, 64, 128, 256])
        windowed = kind != "append" and rng.random() < 0.4
        window, sinks = (_log(rng, 32, 4096), rng.choice([0, 1, 4, 16])) if windowed else (0, 0)
        if kind == "append":
            seqs, new, past = _log(rng, 1, 64), rng.choice([1, _log(rng, 2, 2048)]), rng.randint(0, 8192)
        elif kind == "decode":
            seqs, new, past = _log(rng, 1, 64), 1, _log(rng, 1, 131072)
        else:
            seqs, new, past = rng.randint(1, 8), _log(rng, 2, 8192), rng.choice([0, _log(rng, 1, 8192)])
        c = _case(None, kind, seqs, new, past, heads, page, rng.random() < 0.5 and kind == "append", window, sinks)
        cached = seqs * (new + past) * heads[1] * heads[2]
        # no more than the largest listed case of the kind: rows written, keys read, scores formed by the plain form
        if kind == "append" and (sum(_news(c)) * (heads[0] + 2 * heads[1]) * heads[2] <= 8000 * 80 * 128 and cached <= 1 << 27):
            return c
        if kind == "decode" and cached <= 1 << 28:
            return c
        if kind == "prompt" and seqs * heads[0] * new * (new + past) <= 2 * 32 * 8000 ** 2 and cached <= 1 << 27:
            return c


# ---- lengths: fixed by the case, the longest first, the others spread in a logarithmic scale over a factor of 32 ----
def _spread(n, most, turn):
    return [most if i == 0 else max(min(1, most), int(round(most * 32.0 ** -((i * turn) % 1.0)))) for i in range(n)]


def _news(c):
    return _spread(c["seqs"], c["new"], 0.6180339887)


def _pasts(c):
    # every second sequence of a batch of prompts starts from nothing
    p = _spread(c["seqs"], c["past"], 0.7548776662)
    return [0 if c["kind"] == "prompt" and i % 2 else v for i, v in enumerate(p)]


def _kv_lens(c):
    # a decoding sequence's new token is in the cache already
    return [max(1, p) if c["kind"] == "decode" else p + n for p, n in zip(_pasts(c), _news(c))]


def _pairs(c):
    """Visible (query token, key) pairs of all sequences, and the keys that any query of a sequence sees."""
    pairs = keys = 0
    for n, length in zip(_news(c), _kv_lens(c)):
        first = length - n
        w, s = (c["window"], c["sinks"]) if c["window"] else (length, 0)
        pairs += sum(min(p + 1, w) + max(0, min(s, p + 1 - w)) for p in range(first, length))
        lo = max(0, first - w + 1)
        keys += length - lo + min(s, lo)
    return pairs, keys


def work(case):
    c, rows = case, sum(_news(case))
    q_row, kv_row = c["heads"] * c["hd"], c["kv_heads"] * c["hd"]
    if c["kind"] == "append":  # q, k and v of the new tokens in and out; a norm and a rotation are some ten operations
        return {"bytes": rows * (q_row + 2 * kv_row) * 2 * 2, "flops": rows * (q_row + kv_row) * (9 if c["norm"] else 3)}
    pairs, keys = _pairs(c)
    tables = 4 * sum(-(-n // c["page"]) for n in _kv_lens(c))
    return {"bytes": keys * kv_row * 2 * 2 + rows * q_row * 2 * 2 + tables, "flops": 4 * pairs * q_row}


# ---- inputs ---------------------------------------------------------------------------------------------
def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev, dtype=torch.float32).half()  # noqa: E731
    news, lens = _news(c), _kv_lens(c)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    counts = [-(-n // c["page"]) for n in lens]
    pool = torch.randperm(sum(counts) + 3, generator=g, device=dev).to(torch.int32)  # three pages belong to nobody
    table = torch.full((c["seqs"], max(counts) + 1), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = pool[at: at + n]
        at += n
    shape = (pool.numel(), c["kv_heads"], c["page"], c["hd"])
    # a new cache is cleared memory, and what earlier tokens hold there the append never looks at
    pages = (lambda: torch.zeros(shape, dtype=torch.float16, device=dev)) if c["kind"] == "append" else lambda: normal(*shape)
    s = SimpleNamespace(case=c, rows=starts[-1], max_new=max(news), table=table, K=pages(), V=pages(),
                        kv_len=torch.tensor(lens, dtype=torch.int32, device=dev),
                        q_start=torch.tensor(starts, dtype=torch.int32, device=dev) if max(news) > 1 else None,
                        q_gain=None, k_gain=None)
    if c["kind"] == "append":
        s.qkv = normal(s.rows, (c["heads"] + 2 * c["kv_heads"]) * c["hd"])
        if c["norm"]:
            s.q_gain, s.k_gain = (1 + 0.1 * normal(c["hd"]) for _ in range(2))
        s.out = torch.empty((s.rows, c["heads"] * c["hd"]), dtype=torch.float16, device=dev)
    else:
        s.q = normal(s.rows, c["heads"] * c["hd"]) * 2  # scores of a standard deviation of two: some keys stand out
        s.out = torch.empty_like(s.q)
    if own:
        from paper_2504_08378_amd import binding as B
        s.cache = B.PagedCache(s.K, s.V)
        s.batch = B.PagedBatch(s.table, s.kv_len, s.q_start, s.rows, s.max_new)
        _context(s.table.get_device())
    return s


_contexts = {}  # (device, its stream): a program keeps a context, with its workspace, for each stream that it calls from


def _context(device):
    """The context of the current stream, whose calls lie in order with the fills and reads there."""
    key = device, torch._C._cuda_getCurrentRawStream(device)  # the public form takes 2.5 us, the smallest calls 6
    if key not in _contexts:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a stream's first pass has to run before one is captured: it makes the workspace")
        from paper_2504_08378_amd import binding as B
        _contexts[key] = B.Context(device, stream=torch.cuda.current_stream(device))
    return _contexts[key]


# ---- one pass -------------------------------------------------------------------------------------------
def run(state):
    s, c = state, state.case
    if own:
        context = _context(s.table.get_device())
        if c["kind"] == "append":
            context.paged_append(s.cache, s.batch, s.qkv, s.out, c["heads"], rope_theta=THETA, q_gain=s.q_gain,
                                 k_gain=s.k_gain, eps=EPS)
            return {"q": s.out, "k_pages": s.K, "v_pages": s.V}
        context.paged_attention(s.cache, s.batch, s.q, s.out, c["heads"], window=c["window"], n_sink=c["sinks"])
        return s.out
    return _append(s, c) if c["kind"] == "append" else _attend(s, c)


def _rows(s):
    """Sequence of each row, its place among the sequence's new tokens, and its place in the cache."""
    t = torch.arange(s.rows, device=s.table.device)
    if s.q_start is None:
        return t, torch.zeros_like(t), s.kv_len.long() - 1
    b = torch.searchsorted(s.q_start[1:].contiguous(), t.int(), right=True)
    i = t - s.q_start[b]
    return b, i, s.kv_len[b] - (s.q_start[b + 1] - s.q_start[b]) + i


def _append(s, c):
    h, kv, hd = c["heads"], c["kv_heads"], c["hd"]
    b, _, pos = _rows(s)
    x = s.qkv.view(s.rows, h + 2 * kv, hd)
    qk = x[:, : h + kv].float()
    if s.q_gain is not None:
        gain = torch.cat([s.q_gain.float().expand(h, hd), s.k_gain.float().expand(kv, hd)])
        qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    angle = pos.double()[:, None] * THETA ** (-2.0 * torch.arange(hd // 2, device=x.device, dtype=torch.float64) / hd)
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    lo, hi = qk[..., : hd // 2], qk[..., hd // 2:]
    qk = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).half()
    page, slot = s.table[b, pos // c["page"]].long(), pos % c["page"]
    s.K[page, :, slot] = qk[:, h:]
    s.V[page, :, slot] = x[:, h + kv:]
    return {"q": qk[:, :h].reshape(s.rows, h * hd), "k_pages": s.K, "v_pages": s.V}


def _attend(s, c):
    h, kv, hd, n = c["heads"], c["kv_heads"], c["hd"], s.max_new
    seqs, pages = s.table.shape
    length = pages * c["page"]
    spread = lambda t: t[s.table.clamp(min=0).long()].transpose(1, 2).reshape(seqs, kv, length, hd).float()  # noqa: E731
    K, V = spread(s.K), spread(s.V)
    b, i, _ = _rows(s)
    start = torch.arange(seqs + 1, device=b.device) if s.q_start is None else s.q_start.long()
    count = start[1:] - start[:-1]
    i_all = torch.arange(n, device=b.device)
    q = s.q[(start[:-1, None] + i_all).clamp(max=s.rows - 1)].float().view(seqs, n, kv, h // kv, hd)
    q = q.permute(0, 2, 3, 1, 4).reshape(seqs, kv, -1, hd)  # rows: query head of the key head, token
    score = (torch.matmul(q, K.transpose(2, 3).contiguous()) / math.sqrt(hd)).view(seqs, kv, h // kv, n, length)
    p = (s.kv_len[:, None] - count[:, None] + i_all)[:, :, None]
    j = torch.arange(length, device=b.device)
    see = j <= p
    if c["window"]:
        see = see & ((j > p - c["window"]) | (j < c["sinks"]))
    score = score.masked_fill(~see[:, None, None], -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.matmul(e.view(seqs, kv, -1, length), V).view(seqs, kv, h // kv, n, hd) / e.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4)[b, i].reshape(s.rows, h * hd).half()


# ---- the same in 64 bits, sequence by sequence -----------------------------------------------------------
def exact(case, seed):
    c, s = case, prepare(case, seed)
    h, kv, hd, page = c["heads"], c["kv_heads"], c["hd"], c["page"]
    dev = s.table.device
    f64 = torch.float64
    news, lens, row = _news(c), _kv_lens(c), 0
    if c["kind"] == "append":
        K, V = s.K.to(f64), s.V.to(f64)
        q_out = torch.empty((s.rows, h * hd), dtype=f64, device=dev)
        freq = torch.tensor([THETA ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=f64, device=dev)
        for b, (n, length) in enumerate(zip(news, lens)):
            place = torch.arange(length - n, length, device=dev)
            x = s.qkv[row: row + n].to(f64).view(n, h + 2 * kv, hd)
            parts = [x[:, :h], x[:, h: h + kv]]
            if c["norm"]:
                parts = [y / (y.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w.to(f64)
                         for y, w in zip(parts, (s.q_gain, s.k_gain))]
            turn = torch.polar(torch.ones(n, hd // 2, dtype=f64, device=dev), place.to(f64)[:, None] * freq)[:, None]
            z = [torch.complex(y[..., : hd // 2].contiguous(), y[..., hd // 2:].contiguous()) * turn for y in parts]
            q, k = (torch.cat([w.real, w.imag], -1) for w in z)
            q_out[row: row + n] = q.reshape(n, h * hd)
            at = s.table[b].long()[place // page]
            K[at, :, place % page] = k
            V[at, :, place % page] = x[:, h + kv:]
            row += n
        return {"q": q_out, "k_pages": K, "v_pages": V}
    out = torch.empty((s.rows, h, hd), dtype=f64, device=dev)
    for b, (n, length) in enumerate(zip(news, lens)):
        mine = s.table[b, : -(-length // page)].long()
        place = torch.arange(length - n, length, device=dev)[:, None]
        key = torch.arange(length, device=dev)[None]
        hidden = key > place
        if c["window"]:
            hidden |= (place - key >= c["window"]) & (key >= c["sinks"])
        for head in range(h):
            of = head * kv // h
            k = s.K[mine, of].reshape(-1, hd)[:length].to(f64)
            v = s.V[mine, of].reshape(-1, hd)[:length].to(f64)
            y = s.q[row: row + n, head * hd: (head + 1) * hd].to(f64)
            z = y.mm(k.t().contiguous()).div_(hd ** 0.5).masked_fill_(hidden, -math.inf)
            out[row: row + n, head] = torch.softmax(z, 1).mm(v)
        row += n
    return out.view(s.rows, h * hd)
