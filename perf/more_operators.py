"""Operators of chunks over a bounded cache: the calls that are measured.

New tokens attend to a paged key/value cache under a mask - causal by groups (tokens, or the tokens of a frame), a
sliding window, the first tokens always seen - and give each row's log-sum-exp (kind "attention"); the weight that
their softmax gives to every cached key is summed over rows and heads (kind "weights"); and a cache that has grown
too long keeps its heaviest tokens, packed into its first pages (kind "evict").

``own`` false: elementary torch operations in 32 bits.  ``own`` true: the framework's entry points.
Cases whose lengths differ from sequence to sequence derive them from plain numbers of the case (``_spread``).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # the tiny float32 model (4 heads of 32, chunks of 64 tokens in frames of 16), three branches
        dict(name="attention-tiny-f32", kind="attention", dtype="f32", heads=4, kv_heads=4, d=32, page=16, prefix=64,
             drop=0, branches=3, new_lo=64, new_hi=64, own_lo=0, own_hi=0, group=16, window=0, sinks=0),
        # 16 branches decode a token each behind two multi-camera chunks, over the last 4096 tokens and the first 64
        dict(name="attention-window-single-tokens", kind="attention", dtype="bf16", heads=12, kv_heads=12, d=128,
             page=64, prefix=14040, drop=0, branches=16, new_lo=1, new_hi=1, own_lo=0, own_hi=300, group=1,
             window=4096, sinks=64),
        # ragged causal chunks, four query heads to a key head, a history whose oldest tokens were dropped inside a page
        dict(name="attention-causal-ragged", kind="attention", dtype="bf16", heads=16, kv_heads=4, d=64, page=16,
             prefix=4101, drop=5, branches=13, new_lo=1, new_hi=1501, own_lo=0, own_hi=777, group=1, window=0, sinks=0),
        # a multi-camera chunk of three frames (6 x 390 tokens each) behind two chunks
        dict(name="attention-frames-multi-camera", kind="attention", dtype="bf16", heads=12, kv_heads=12, d=128,
             page=64, prefix=14040, drop=0, branches=1, new_lo=7020, new_hi=7020, own_lo=0, own_hi=0, group=2340,
             window=0, sinks=0),
        # a history of two chunks of the larger model (12096 tokens, 16 heads of 128) filled in at once, causal
        dict(name="attention-causal-long", kind="attention", dtype="bf16", heads=16, kv_heads=16, d=128, page=256,
             prefix=0, drop=0, branches=1, new_lo=24192, new_hi=24192, own_lo=0, own_hi=0, group=1, window=0, sinks=0),
        # the tiny float32 model: the call's latency counts
        dict(name="weights-tiny-f32", kind="weights", dtype="f32", heads=4, kv_heads=4, d=32, page=16, prefix=64,
             drop=0, branches=3, new_lo=64, new_hi=64, own_lo=0, own_hi=0, group=16, window=0, sinks=0, decay=1.0),
        # what 16 decoded tokens look at in the history that they share
        dict(name="weights-single-tokens", kind="weights", dtype="bf16", heads=12, kv_heads=12, d=128, page=64,
             prefix=14040, drop=0, branches=16, new_lo=1, new_hi=1, own_lo=0, own_hi=300, group=1, window=0, sinks=0,
             decay=1.0),
        # ragged causal chunks with shared key heads, older weight fading
        dict(name="weights-causal-ragged", kind="weights", dtype="bf16", heads=16, kv_heads=4, d=64, page=16,
             prefix=4101, drop=5, branches=13, new_lo=1, new_hi=1501, own_lo=0, own_hi=777, group=1, window=0, sinks=0,
             decay=0.75),
        # a whole multi-camera chunk over three chunks of keys, the first block of a pass
        dict(name="weights-multi-camera", kind="weights", dtype="bf16", heads=12, kv_heads=12, d=128, page=64,
             prefix=14040, drop=0, branches=1, new_lo=7020, new_hi=7020, own_lo=0, own_hi=0, group=2340, window=0,
             sinks=0, decay=0.0),
        # the single-camera model (8 blocks, 8 heads of 64, chunks of 768): a window of three chunks back to two
        dict(name="evict-single-camera", kind="evict", dtype="bf16", blocks=8, kv_heads=8, d=64, page=64, parent=2304,
             children=0, step=0, keep=1536, sinks=16, recent=768),
        # twelve futures of one history in the multi-camera model: each keeps its own choice of the shared pages
        dict(name="evict-branches", kind="evict", dtype="bf16", blocks=20, kv_heads=12, d=128, page=64, parent=1130,
             children=12, step=130, keep=901, sinks=130, recent=260),
        # the multi-camera model's window: three chunks of 7020 tokens back to two, the newest one whole
        dict(name="evict-multi-camera", kind="evict", dtype="bf16", blocks=20, kv_heads=12, d=128, page=64,
             parent=21060, children=0, step=0, keep=14040, sinks=64, recent=7020),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))

    kind = rng.choice(["attention", "attention", "weights", "weights", "evict"])
    f32 = rng.random() < 0.2
    d = rng.choice([32, 64, 128] if f32 else [64, 128])
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    c = dict(kind=kind, dtype="f32" if f32 else "bf16", kv_heads=kv, d=d, page=rng.choice([16, 32, 64, 128, 256]))
    if kind == "evict":
        c.update(blocks=log(1, 20), parent=log(2, 21060), children=rng.choice([0, 0, log(1, 16)]), step=0, keep=0,
                 sinks=0, recent=0)
        if c["children"]:
            c.update(step=log(1, 200))
        while _pool_bytes(c) > 2.5e9:
            c["blocks"] = max(1, c["blocks"] // 2)
            c["children"] = c["children"] * 2 // 3
            c["parent"] = max(2, c["parent"] * 2 // 3)
        c["step"] *= c["children"] > 0
        n = c["parent"] + c["step"]
        c["keep"] = rng.randint(0, n)
        c["sinks"] = rng.choice([0, rng.randint(0, c["keep"]) // 8])
        c["recent"] = rng.choice([0, rng.randint(0, c["keep"] - c["sinks"])])
        return c
    heads = kv * (rng.choice([1, 1, 2, 4, 8]) if kv <= 4 else 1)
    lo, hi = sorted((log(1, 7020), log(1, 7020)))
    if rng.random() < 0.4:
        lo, hi = 1, rng.choice([1, 1, 5])
    c.update(heads=heads, branches=log(1, 32), new_lo=lo, new_hi=hi, prefix=rng.choice([0, log(1, 30000)]), drop=0,
             own_lo=0, own_hi=log(1, 1000), group=rng.choice([0, 1, 1, log(1, 2400)]), window=0, sinks=0)
    if c["prefix"]:
        c["drop"] = rng.randint(0, min(c["page"], c["prefix"]) - 1)
    if rng.random() < 0.4:
        c.update(window=log(1, 10000), sinks=rng.choice([0, log(1, 300)]))
    if kind == "weights":
        c["decay"] = rng.choice([0.0, 0.5, 1.0])
    while _pairs(c) * c["heads"] * 4 * d > (1e11 if f32 else 1.2e12) or _pool_bytes(c) > 8e8:
        c["branches"] = max(1, c["branches"] * 2 // 3)
        c["new_hi"] = max(1, c["new_hi"] * 2 // 3)
        c["new_lo"] = min(c["new_lo"], c["new_hi"])
        if c["prefix"]:
            c["prefix"] = max(c["drop"] + 1, c["prefix"] * 2 // 3)
    return c


def _spread(lo, hi, n, salt):
    """n lengths in [lo, hi], fixed by the case alone."""
    return [lo + (i * 7919 + salt * 104729) % (hi - lo + 1) for i in range(n)]


def _lengths(case):
    """Per sequence: its own earlier tokens and its new tokens."""
    n = case["branches"]
    return _spread(case["own_lo"], case["own_hi"], n, 2), _spread(case["new_lo"], case["new_hi"], n, 1)


def _tokens(case):
    """Per sequence: all its tokens."""
    return [case["prefix"] - case["drop"] + b + n for b, n in zip(*_lengths(case))]


def _ceil(a, b):
    return -(-a // b)


def _n_pages(case):
    """Pages of the case's pool: what its sequences need, with every last page private, and a few more."""
    page = case["page"]
    if case["kind"] == "evict":
        if not case["children"]:
            return _ceil(case["parent"], page) + 2
        return (case["children"] * 2 + 1) * (_ceil(case["parent"] + case["step"], page) + 1)
    before, new = _lengths(case)
    return _ceil(case["prefix"], page) + sum(_ceil(b + n, page) + 2 for b, n in zip(before, new)) + 2


def _pool_bytes(case):
    e = 2 if case["dtype"] == "bf16" else 4
    return 2 * case.get("blocks", 1) * _n_pages(case) * case["page"] * case["kv_heads"] * case["d"] * e


def _seen(case, tokens, new, xp):
    """Of the last `new` of `tokens` tokens: the windows [begin, end) that they see besides the first `sinks`."""
    r = xp.arange(new)
    g = case["group"] or new
    end = tokens - new + xp.minimum((r // g + 1) * g, xp.full_like(r, new))
    begin = (end - case["window"]) * (end > case["window"]) if case["window"] else 0 * end
    return begin, end


def _pairs(case):
    """Visible (row, key) pairs, over all sequences."""
    total = 0
    for t, n in zip(_tokens(case), _lengths(case)[1]):
        begin, end = _seen(case, t, n, np)
        total += int((end - begin + np.minimum(begin, case["sinks"])).sum())
    return total


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    d, kv = case["d"], case["kv_heads"]
    if case["kind"] == "evict":
        seqs, tokens = max(1, case["children"]), case["parent"] + case["step"]
        # a token's row in every block, key and value; the first tokens stay
        row = 2 * case["blocks"] * kv * d * e
        moved = case["keep"] - case["sinks"] if case["keep"] < tokens else 0
        return {"bytes": seqs * (2 * row * moved + 8 * tokens + 4 * case["keep"]), "flops": 0}
    tokens, (_, new) = _tokens(case), _lengths(case)
    rows, heads, shared = sum(new), case["heads"], case["prefix"] - case["drop"]
    keys = shared + sum(t - shared for t in tokens)
    if case["window"]:  # what no row sees is not read
        keys = min(keys, sum(min(t, case["window"] + n + case["sinks"]) for t, n in zip(tokens, new)))
    flops = _pairs(case) * heads * d
    if case["kind"] == "attention":
        return {"bytes": e * (2 * keys * kv * d + 2 * rows * heads * d) + 4 * rows * heads, "flops": 4 * flops}
    old = 1 if case["decay"] else 0
    return {"bytes": e * (keys * kv * d + rows * heads * d) + 4 * rows * heads + 4 * (1 + old) * sum(tokens),
            "flops": 2 * flops}


# ---------------------------------------------------------------- the cache's bookkeeping, plain

class Pages:
    """Page tables over key and value buffers [blocks, pages, kv_heads, page, d]: sequences share pages by
    reference; the lowest free page (and sequence number) is taken first."""

    def __init__(self, keys, values, page, n_pages, max_seqs):
        self.keys, self.values, self.page = keys, values, page
        self.refs = [0] * n_pages
        self.seqs = [None] * max_seqs

    def new(self):
        s = self.seqs.index(None)
        self.seqs[s] = [0, 0, []]
        return s

    def _take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def fork(self, seq, n):
        out = []
        for _ in range(n):
            s = self.new()
            first, tokens, pages = self.seqs[seq]
            self.seqs[s] = [first, tokens, list(pages)]
            for p in pages:
                self.refs[p] += 1
            out.append(s)
        return out

    def extend(self, seqs, tokens):
        copies = []
        for s, n in zip(seqs, tokens):
            first, have, pages = self.seqs[s]
            used = (first + have) % self.page
            if n and used and self.refs[pages[-1]] > 1:
                p = self._take()
                copies.append((pages[-1], p, used))
                self.refs[pages[-1]] -= 1
                pages[-1] = p
            while len(pages) * self.page < first + have + n:
                pages.append(self._take())
            self.seqs[s][1] = have + n
        if self.keys is not None:
            # one source and one row count at a time: the children of one parent share both
            for src, used in sorted({(a, u) for a, _, u in copies}):
                dst = torch.tensor([b for a, b, u in copies if (a, u) == (src, used)], device=self.keys.device)
                for buf in (self.keys, self.values):
                    buf[:, dst, :, :used] = buf[:, src:src + 1, :, :used]

    def trim(self, seq, front):
        first, tokens, pages = self.seqs[seq]
        first += front
        for p in pages[:first // self.page]:
            self.refs[p] -= 1
        self.seqs[seq] = [first % self.page, tokens - front, pages[first // self.page:]]

    def free(self, seqs):
        for s in seqs:
            for p in self.seqs[s][2]:
                self.refs[p] -= 1
            self.seqs[s] = None

    def evict(self, seqs, keep, weights, kept, sinks, recent):
        """seqs[i] keeps keep[i] tokens: the first `sinks`, the last `recent` and the heaviest of the others by
        weights[i] (the lowest index first among equals), in their order, from its first place on.  Pages that only it
        holds are filled in place, shared ones replaced; weights follow, those past the kept ones become 0."""
        before, gone = list(self.refs), []
        new, src, dst = [], [], []
        for i, (s, k) in enumerate(zip(seqs, keep)):
            first, tokens, pages = self.seqs[s]
            k = min(k, tokens)
            w = weights[i, :tokens]
            mid = torch.sort(w[sinks:tokens - recent], descending=True, stable=True)[1][:max(0, k - sinks - recent)]
            at = torch.arange(tokens, device=w.device)
            at = torch.cat((at[:sinks], mid.sort()[0] + sinks, at[tokens - recent:])) if k < tokens else at
            kept[i, :k] = at
            if k == tokens:
                new.append(None)
                continue
            w[:k], w[k:] = w[at], 0.0
            n = _ceil(first + k, self.page) if k else 0
            table = [p if before[p] == 1 or (j + 1) * self.page <= first + sinks else self._take()
                     for j, p in enumerate(pages[:n])]
            gone += [p for j, p in enumerate(pages) if j >= n or table[j] != p]
            new.append([first if k else 0, k, table])
            old, now = (torch.tensor(t, dtype=torch.long, device=w.device) for t in (pages, table))
            a, b = first + at, first + torch.arange(k, device=w.device)
            src.append((old[a // self.page], a % self.page))
            dst.append((now[b // self.page], b % self.page))
        for s, t in zip(seqs, new):
            if t is not None:
                self.seqs[s] = t
        for p in gone:
            self.refs[p] -= 1
        if src:
            (a, i), (b, j) = ([torch.cat(x) for x in zip(*y)] for y in (src, dst))
            for buf in (self.keys, self.values):
                buf[:, b, :, j] = buf[:, a, :, i]

    def pages(self, seq):
        first, tokens, pages = self.seqs[seq]
        return first, tokens, np.array(pages, np.int32)


def _pool(case, keys, values, max_seqs):
    if own:
        from paper_2604_20289_amd import xcache
        return xcache.Pool(keys, values, q_heads=case.get("heads", case["kv_heads"]), max_seqs=max_seqs,
                           stream=torch.cuda.current_stream().cuda_stream)
    return Pages(keys, values, case["page"], keys.shape[1], max_seqs)


def _branches(pool, case):
    """The case's sequences: a parent with the shared history, its oldest tokens dropped, forked; then the
    branches grow in three turns, so that their pages lie between each other's."""
    before, new = _lengths(case)
    parent = pool.new()
    if case["prefix"]:
        pool.extend([parent], [case["prefix"]])
        if case["drop"]:
            pool.trim(parent, front=case["drop"])
    seqs = pool.fork(parent, case["branches"])
    total = [b + n for b, n in zip(before, new)]
    for turn in range(3):
        pool.extend(seqs, [t * (turn + 1) // 3 - t * turn // 3 for t in total])
    pool.free([parent])
    return seqs, new


# ---------------------------------------------------------------- inputs

def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)

    kv, d = case["kv_heads"], case["d"]
    shape = (_n_pages(case), kv, case["page"], d)
    x = {}
    for name in ("keys", "values"):
        x[name] = torch.empty((case.get("blocks", 1), *shape), dtype=dt, device="cuda")
        for b in range(len(x[name])):
            x[name][b] = normal(*shape)
    if case["kind"] == "evict":
        # weights as attention leaves them: few heavy tokens, and some that nothing looked at
        n, tokens = max(1, case["children"]), case["parent"] + case["step"]
        w = torch.exp(2.0 * torch.randn((n, tokens), generator=g, device="cuda"))
        x["weights"] = w * (torch.rand((n, tokens), generator=g, device="cuda") > 0.1)
        return x
    # normalised queries with gains over 1: a softmax of some sharpness
    x["q"] = normal(sum(_lengths(case)[1]), case["heads"], d, scale=1.5)
    if case["kind"] == "weights":
        x["weights"] = torch.rand((case["branches"], max(_tokens(case)) + 5), generator=g, device="cuda")
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    st = {"case": case, **x}
    n = case["children"] if case["kind"] == "evict" else case["branches"]
    pool = st["pool"] = _pool(case, x["keys"], x["values"], n + 1)
    if case["kind"] == "evict":
        st["parent"] = pool.new()
        pool.extend([st["parent"]], [case["parent"]])
        st["kept"] = torch.zeros((max(1, n), case["parent"] + case["step"]), dtype=torch.int32, device="cuda")
        st["given"] = x["weights"].clone()
        if own:
            from paper_2604_20289_amd import xcache
            st["batch"] = xcache.Batch(pool)
        return st
    seqs, new = _branches(pool, case)
    st["plan"] = _plan(pool, seqs, new, case)
    if case["kind"] == "weights":
        st["lse"] = _lse(st)
    else:
        st["out"] = torch.empty_like(x["q"])
        st["lse"] = torch.empty(x["q"].shape[:2], device="cuda")
    if own:
        from paper_2604_20289_amd import xcache
        st["batch"] = xcache.Batch(pool)
        st["batch"].set_chunk(seqs, new, group=case["group"], window=case["window"], sinks=case["sinks"])
    return st


def _plan(pool, seqs, new, case):
    """(rows, tokens, pages and places in them of the tokens, window begin and end of each row) of each sequence."""
    out, row = [], 0
    for s, n in zip(seqs, new):
        first, tokens, pages = pool.pages(s)
        at = first + np.arange(tokens)
        page, r = (torch.from_numpy(x.astype(np.int64)).to("cuda") for x in (pages[at // case["page"]], at % case["page"]))
        begin, end = _seen(case, tokens, n, np)
        out.append((row, row + n, tokens, page, r, begin, end))
        row += n
    return out


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    if case["kind"] == "evict":
        return _evict(st)
    if case["kind"] == "attention":
        if own:
            st["batch"].chunk_attention(0, st["q"], st["out"], lse=st["lse"])
        else:
            _attention(st)
        return {"out": st["out"], "lse": st["lse"]}
    if own:
        st["batch"].chunk_weights(0, st["q"], st["lse"], st["weights"], decay=case["decay"])
    else:
        _weights(st)
    return st["weights"]


def _evict(st):
    """One chunk of a rollout: its sequences shrink to what they keep, and room is made for the next chunk.  Or, with
    children: they are forked and grow by a step first, and end with the pass."""
    case, pool = st["case"], st["pool"]
    seqs, step, weights = [st["parent"]], case["parent"] - case["keep"], st["weights"]
    if case["children"]:
        seqs = pool.fork(st["parent"], case["children"])
        pool.extend(seqs, [case["step"]] * len(seqs))
        weights.copy_(st["given"])
    (st["batch"] if own else pool).evict(seqs, [case["keep"]] * len(seqs), weights, st["kept"], sinks=case["sinks"],
                                         recent=case["recent"])
    tables = [pool.pages(s) for s in seqs]
    if case["children"]:
        pool.free(seqs)
    else:
        pool.extend(seqs, [step])
    tables = [np.concatenate(([first, tokens], pages)) for first, tokens, pages in tables]
    return {"keys": st["keys"], "values": st["values"], "weights": weights, "kept": st["kept"],
            "tables": np.concatenate(tables)}


def _scores(st, piece, a, b, q, upto):
    """Scores [kv_heads, rows * group, keys] of rows [a, b) of a sequence over its first `upto` tokens, those that a row
    does not see at -infinity."""
    case, (lo, hi, tokens, page, r, begin, end) = st["case"], piece
    kv, d = case["kv_heads"], case["d"]
    group = case["heads"] // kv
    k = st["keys"][0, page[:upto], :, r[:upto]].float().transpose(0, 1)
    q = q[lo + a:lo + b].float().view(b - a, kv, group, d).permute(1, 0, 2, 3).reshape(kv, -1, d)
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
    if begin[a] > 0 or begin[b - 1] > 0 or end[a] < upto:
        j = torch.arange(upto, device="cuda")
        first, last = (torch.from_numpy(x[a:b]).cuda()[:, None] for x in (begin, end))
        hidden = (j >= last) | (j < first) & (j >= case["sinks"])
        s.view(kv, b - a, group, upto).masked_fill_(hidden[:, None], -math.inf)
    return s


def _blocks(st, piece):
    """Rows of a sequence, as many at a time as keep a block of scores near 1 GB, and the tokens they reach to."""
    lo, hi, tokens, end = piece[0], piece[1], piece[2], piece[6]
    step = max(1, (1 << 28) // (st["case"]["heads"] * tokens))
    for a in range(0, hi - lo, step):
        b = min(a + step, hi - lo)
        yield a, b, int(end[b - 1])


def _rows_of(x, kv, rows):
    """[kv, rows * group, n] as [rows, heads, n]."""
    return x.view(kv, rows, -1, x.shape[-1]).transpose(0, 1).reshape(rows, -1, x.shape[-1])


def _attention(st):
    kv = st["case"]["kv_heads"]
    for piece in st["plan"]:
        lo, page, r = piece[0], piece[3], piece[4]
        for a, b, upto in _blocks(st, piece):
            s = _scores(st, piece, a, b, st["q"], upto)
            v = st["values"][0, page[:upto], :, r[:upto]].float().transpose(0, 1).contiguous()
            m = s.amax(-1, keepdim=True)
            p = torch.exp_(s.sub_(m))
            total = p.sum(-1, keepdim=True)
            st["out"][lo + a:lo + b] = _rows_of(torch.matmul(p, v) / total, kv, b - a)
            st["lse"][lo + a:lo + b] = _rows_of(m + torch.log(total), kv, b - a)[..., 0]


def _weights(st):
    case = st["case"]
    kv = case["kv_heads"]
    for i, piece in enumerate(st["plan"]):
        lo, tokens = piece[0], piece[2]
        w = st["weights"][i, :tokens]
        if case["decay"]:
            w *= case["decay"]
        else:
            w.zero_()
        for a, b, upto in _blocks(st, piece):
            s = _scores(st, piece, a, b, st["q"], upto)
            lse = st["lse"][lo + a:lo + b].view(b - a, kv, -1).transpose(0, 1).reshape(kv, -1, 1)
            w[:upto] += torch.exp_(s.sub_(lse)).sum((0, 1))


def _lse(st):
    """The rows' log-sum-exp, as the attention before has given it: an input."""
    kv = st["case"]["kv_heads"]
    out = torch.empty(st["q"].shape[:2], device="cuda")
    for piece in st["plan"]:
        for a, b, upto in _blocks(st, piece):
            x = torch.logsumexp(_scores(st, piece, a, b, st["q"], upto), -1, keepdim=True)
            out[piece[0] + a:piece[0] + b] = _rows_of(x, kv, b - a)[..., 0]
    return out


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    if case["kind"] == "evict":
        return None  # nothing is computed: numbers are chosen and moved
    x = _inputs(case, seed)
    pool = Pages(x["keys"], x["values"], case["page"], x["keys"].shape[1], case["branches"] + 1)
    seqs, new = _branches(pool, case)
    heads, kv, d = case["heads"], case["kv_heads"], case["d"]
    attention = case["kind"] == "attention"
    if attention:
        out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
        lses = torch.empty(out.shape[:2], dtype=torch.float64, device="cuda")
    else:
        given = _lse({"case": case, **x, "plan": _plan(pool, seqs, new, case)}).double()
        weights = x["weights"].double()
    row = 0
    for i, (s, n) in enumerate(zip(seqs, new)):
        first, tokens, pages = pool.pages(s)
        at = torch.arange(first, first + tokens, device="cuda")
        page_of = torch.from_numpy(pages).to("cuda").long()[at // case["page"]]
        j = torch.arange(tokens, device="cuda")
        if not attention:
            weights[i, :tokens] *= case["decay"]
        for h in range(heads):
            k = x["keys"][0, page_of, h * kv // heads, at % case["page"]].double().T.contiguous()
            v = x["values"][0, page_of, h * kv // heads, at % case["page"]].double()
            for lo in range(0, n, 4096):
                r = torch.arange(lo, min(lo + 4096, n), device="cuda")
                # the last token of the row's group, and what is too old for it
                group = case["group"] if case["group"] else n
                last = (tokens - n + (torch.div(r, group, rounding_mode="floor") + 1) * group - 1).clamp(max=tokens - 1)
                sees = j[None] <= last[:, None]
                if case["window"]:
                    sees &= (last[:, None] - j[None] < case["window"]) | (j[None] < case["sinks"])
                z = x["q"][row + r, h].double() @ k / d ** 0.5
                if attention:
                    z = torch.where(sees, z, torch.full_like(z, -math.inf))
                    out[row + r, h] = torch.softmax(z, 1) @ v
                    lses[row + r, h] = torch.logsumexp(z, 1)
                else:
                    weights[i, :tokens] += (torch.exp(z - given[row + r, h][:, None]) * sees).sum(0)
        row += n
    return {"out": out, "lse": lses} if attention else weights
