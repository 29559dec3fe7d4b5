"""Operators of branching rollouts over a paged key/value cache: the calls that are measured.

Many candidate futures branch from one history.  Three kinds of operator serve them: the per-head norms and
rotary positions of new queries and keys, written with the values into the branches' pages (kind "norm_rope"); the attention of the branches' queries over the history they share and their own
tokens (kind "attention"); and the cache's page operators - fork, private copies, free, compaction (kind "pages").

``own`` false: elementary torch operations in 32 bits.  ``own`` true: the framework's entry points.
Cases whose lengths differ from branch to branch derive them from plain numbers of the case (``_spread``).
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
THETA = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # eight branches decoding one token each at the multi-camera width: the call's latency counts
        dict(name="norm-rope-single-tokens", kind="norm_rope", dtype="bf16", heads=12, kv_heads=12, d=128, page=64,
             branches=8, new_lo=1, new_hi=1, axes=3, grid_h=15, grid_w=26),
        # the tiny float32 model (4 heads of 32, 64 tokens a chunk), three branches
        dict(name="norm-rope-tiny-f32", kind="norm_rope", dtype="f32", heads=4, kv_heads=4, d=32, page=16,
             branches=3, new_lo=64, new_hi=64, axes=3, grid_h=4, grid_w=4),
        # ragged text-like branches: shared key heads, one position axis, small pages
        dict(name="norm-rope-ragged-shared-heads", kind="norm_rope", dtype="bf16", heads=16, kv_heads=4, d=64, page=16,
             branches=13, new_lo=1, new_hi=1501, axes=1, grid_h=1, grid_w=1),
        # one multi-camera chunk (7020 tokens, hidden 1536) in each of four branches
        dict(name="norm-rope-multi-camera", kind="norm_rope", dtype="bf16", heads=12, kv_heads=12, d=128, page=64,
             branches=4, new_lo=7020, new_hi=7020, axes=3, grid_h=15, grid_w=26),
        # three branches of the tiny float32 model: 64 new tokens over a shared chunk
        dict(name="attention-tiny-f32", kind="attention", dtype="f32", heads=4, kv_heads=4, d=32, page=16, prefix=64,
             drop=0, branches=3, new_lo=64, new_hi=64, own_lo=0, own_hi=0),
        # 16 branches, one token each, behind two multi-camera chunks of shared history
        dict(name="attention-single-tokens", kind="attention", dtype="bf16", heads=12, kv_heads=12, d=128, page=64,
             prefix=14040, drop=0, branches=16, new_lo=1, new_hi=1, own_lo=0, own_hi=300),
        # 64 branches, one token each, behind three chunks of the larger model (12096 tokens, 16 heads of 128)
        dict(name="attention-single-tokens-long", kind="attention", dtype="bf16", heads=16, kv_heads=16, d=128,
             page=256, prefix=36288, drop=0, branches=64, new_lo=1, new_hi=1, own_lo=100, own_hi=900),
        # ragged lengths, four queries heads to a key head, a history whose oldest tokens were dropped inside a page
        dict(name="attention-ragged-shared-heads", kind="attention", dtype="bf16", heads=16, kv_heads=4, d=64, page=16,
             prefix=4101, drop=5, branches=13, new_lo=1, new_hi=201, own_lo=0, own_hi=777),
        # the single-camera model (768 tokens, 8 heads of 64): one chunk in each of eight branches
        dict(name="attention-single-camera", kind="attention", dtype="bf16", heads=8, kv_heads=8, d=64, page=64,
             prefix=1536, drop=0, branches=8, new_lo=768, new_hi=768, own_lo=0, own_hi=0),
        # the multi-camera model: one chunk in each of four branches, two chunks of shared history
        dict(name="attention-multi-camera", kind="attention", dtype="bf16", heads=12, kv_heads=12, d=128, page=64,
             prefix=14040, drop=0, branches=4, new_lo=7020, new_hi=7020, own_lo=0, own_hi=0),
        # 16 children of a two-chunk history in the single-camera model's 8 blocks: each gets its own last page
        dict(name="pages-fork", kind="pages", dtype="bf16", blocks=8, kv_heads=8, d=64, page=64, parent=1573,
             children=16, rounds=1, step=1, keep=0),
        # a search step over the multi-camera model's 20 blocks: twelve futures grow in turn, four survive, and the
        # pool is compacted
        dict(name="pages-search-step", kind="pages", dtype="bf16", blocks=20, kv_heads=12, d=128, page=64, parent=1130,
             children=12, rounds=3, step=130, keep=4),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))

    kind = rng.choice(["norm_rope", "attention", "attention", "pages"])
    f32 = rng.random() < 0.2
    d = rng.choice([32, 64, 128] if f32 else [64, 128])
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    group = rng.choice([1, 1, 2, 4]) if kv <= 4 else 1
    c = dict(kind=kind, dtype="f32" if f32 else "bf16", kv_heads=kv, d=d, page=rng.choice([16, 32, 64, 128, 256]))
    if kind == "pages":
        c.update(blocks=log(1, 20), parent=log(1, 7020), children=log(1, 24), rounds=rng.choice([1, 1, 2, 3]),
                 step=log(1, 150), keep=0)
        c["keep"] = rng.randint(0, c["children"])
        while work(c)["bytes"] > 3.5e8 or _pool_bytes(c) > 9e8:
            c["blocks"] = max(1, c["blocks"] // 2)
            c["children"] = max(1, c["children"] * 2 // 3)
            c["parent"] = max(1, c["parent"] * 2 // 3)
            c["keep"] = min(c["keep"], c["children"])
        return c
    c.update(heads=kv * group, branches=log(1, 64))
    lo, hi = sorted((log(1, 7020), log(1, 7020)))
    if kind == "norm_rope":
        c.update(new_lo=lo, new_hi=hi, axes=rng.choice([1, 3]), grid_h=rng.randint(1, 20), grid_w=rng.randint(1, 40))
        while work(c)["bytes"] > 5e8:
            c["branches"] = max(1, c["branches"] // 2)
            c["new_hi"] = max(c["new_lo"], c["new_hi"] * 2 // 3)
            c["new_lo"] = max(1, c["new_lo"] * 2 // 3)
        return c
    if rng.random() < 0.4:
        lo, hi = 1, rng.choice([1, 1, 4])
    c.update(new_lo=lo, new_hi=hi, prefix=log(1, 48000), drop=0, own_lo=0, own_hi=log(1, 1000))
    c["drop"] = rng.randint(0, min(c["page"], c["prefix"]) - 1)
    while work(c)["flops"] > (1e11 if f32 else 2e12) or _pool_bytes(c) > 8e8:
        c["branches"] = max(1, c["branches"] * 2 // 3)
        c["new_hi"] = max(1, c["new_hi"] * 2 // 3)
        c["new_lo"] = min(c["new_lo"], c["new_hi"])
        c["prefix"] = max(c["drop"] + 1, c["prefix"] * 2 // 3)
    return c


def _spread(lo, hi, n, salt):
    """n lengths in [lo, hi], fixed by the case alone."""
    return [lo + (i * 7919 + salt * 104729) % (hi - lo + 1) for i in range(n)]


def _lengths(case):
    """Per branch: its own earlier tokens and its new tokens."""
    n = case["branches"]
    new = _spread(case["new_lo"], case["new_hi"], n, 1)
    if case["kind"] == "norm_rope":
        return [0] * n, new
    return _spread(case["own_lo"], case["own_hi"], n, 2), new


def _ceil(a, b):
    return -(-a // b)


def _n_pages(case):
    """Pages of the case's pool: what its sequences need, with every last page private, and a few more."""
    page = case["page"]
    if case["kind"] == "pages":
        grown = case["rounds"] * case["step"]
        return _ceil(case["parent"], page) + case["children"] * (_ceil(grown, page) + 1) + 2
    before, new = _lengths(case)
    prefix = case.get("prefix", 0)
    return _ceil(prefix, page) + sum(_ceil(b + n, page) + 2 for b, n in zip(before, new)) + 2


def _pool_bytes(case):
    e = 2 if case["dtype"] == "bf16" else 4
    return 2 * case.get("blocks", 1) * _n_pages(case) * case["page"] * case["kv_heads"] * case["d"] * e


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    d, kv = case["d"], case["kv_heads"]
    if case["kind"] == "pages":
        # a token's row in every block, key and value
        row = 2 * case["blocks"] * kv * d * e
        tail = case["parent"] % case["page"]
        copied = tail * (case["children"] + 1) if tail else 0
        return {"bytes": row * (copied + 2 * case["page"] * _plan_moves(case)), "flops": 0}
    before, new = _lengths(case)
    rows, heads = sum(new), case["heads"]
    if case["kind"] == "norm_rope":
        elems = rows * (heads + 2 * kv) * d
        return {"bytes": 2 * e * elems + rows * 4 * case["axes"] + 8 * d, "flops": 10 * rows * (heads + kv) * d}
    shared = case["prefix"] - case["drop"]
    keys = shared + sum(before) + rows
    flops = sum(4 * d * heads * n * (shared + b + n) for b, n in zip(before, new))
    return {"bytes": e * (2 * keys * kv * d + 2 * rows * heads * d), "flops": flops}


def _plan_moves(case):
    """Pages that the compaction of a "pages" case moves."""
    return _grow_and_prune(Pages(None, None, case["page"], _n_pages(case), case["children"] + 1), case,
                           start=True)[1]


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

    def trim(self, seq, front=0, back=0):
        first, tokens, pages = self.seqs[seq]
        first, tokens = first + front, tokens - front - back
        gone = pages[:first // self.page] if tokens else pages
        pages = pages[len(gone):]
        first = first % self.page if tokens else 0
        need = _ceil(first + tokens, self.page) if tokens else 0
        gone = gone + pages[need:]
        for p in gone:
            self.refs[p] -= 1
        self.seqs[seq] = [first, tokens, pages[:need]]

    def free(self, seqs):
        for s in seqs:
            for p in self.seqs[s][2]:
                self.refs[p] -= 1
            self.seqs[s] = None

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r]
        src = [p for p in live if p >= len(live)]
        dst = [p for p, r in enumerate(self.refs[:len(live)]) if not r]
        if src and self.keys is not None:
            a, b = (torch.tensor(x, device=self.keys.device) for x in (src, dst))
            for buf in (self.keys, self.values):
                buf[:, b] = buf[:, a]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for s in self.seqs:
            if s is not None:
                s[2] = [to.get(p, p) for p in s[2]]
        return len(src)

    def pages(self, seq):
        first, tokens, pages = self.seqs[seq]
        return first, tokens, np.array(pages, np.int32)


def _pool(case, keys, values, max_seqs):
    if own:
        from paper_2604_20289_amd import xcache
        return xcache.Pool(keys, values, q_heads=case.get("heads", case["kv_heads"]), max_seqs=max_seqs,
                           stream=torch.cuda.current_stream().cuda_stream)
    return Pages(keys, values, case["page"], keys.shape[1], max_seqs)


def _grow_and_prune(pool, case, start=False):
    """One pass of a "pages" case: fork, grow in turns, free all but the survivors, compact.  Returns the survivors'
    tables and the number of pages moved, and leaves the pool as it found it (its parent is sequence 0)."""
    if start:
        pool.extend([pool.new()], [case["parent"]])
    kids = pool.fork(0, case["children"])
    for _ in range(case["rounds"]):
        pool.extend(kids, [case["step"]] * len(kids))
    kept = [k for i, k in enumerate(kids) if (i + 1) * case["keep"] // len(kids) > i * case["keep"] // len(kids)]
    pool.free([k for k in kids if k not in kept])
    moved = pool.compact()
    tables = [pool.pages(k) for k in kept]
    pool.free(kept)
    return tables, moved


def _branches(pool, case):
    """The case's branches: a parent with the shared history, its oldest tokens dropped, forked; then the
    branches grow in three turns, so that their pages lie between each other's."""
    before, new = _lengths(case)
    parent = pool.new()
    if case.get("prefix"):
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
    shape = (case.get("blocks", 1), _n_pages(case), kv, case["page"], d)
    x = {"keys": normal(*shape), "values": normal(*shape)}
    if case["kind"] == "pages":
        return x
    rows = sum(_lengths(case)[1])
    if case["kind"] == "attention":
        # normalised queries with gains over 1: a softmax of some sharpness
        x["q"] = normal(rows, case["heads"], d, scale=1.5)
        return x
    x["qkv"] = normal(rows, (case["heads"] + 2 * kv) * d, scale=2.0)
    x["gq"] = 1.0 + 0.25 * torch.randn(d, generator=g, device="cuda")
    x["gk"] = 1.0 + 0.25 * torch.randn(d, generator=g, device="cuda")
    # tokens of a branch count through their grids from a frame of their own, far into a rollout
    pos = []
    for i, n in enumerate(_lengths(case)[1]):
        t = torch.arange(n, device="cuda")
        base = 1000 * (seed % 97) + 50021 * i
        if case["axes"] == 1:
            pos.append((base + t)[:, None])
        else:
            w, hw = case["grid_w"], case["grid_h"] * case["grid_w"]
            pos.append(torch.stack((base + t // hw, t % hw // w, t % w), 1))
    x["positions"] = torch.cat(pos).to(torch.int32)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    st = {"case": case, **x}
    n = case.get("children", case.get("branches"))
    pool = st["pool"] = _pool(case, x["keys"], x["values"], n + 1)
    if case["kind"] == "pages":
        pool.extend([pool.new()], [case["parent"]])
        return st
    seqs, new = _branches(pool, case)
    if own:
        from paper_2604_20289_amd import xcache
        st["batch"] = xcache.Batch(pool)
        st["batch"].set(seqs, new)
    else:
        # (rows, first token's place in the pages, keys, page table) of each branch
        st["plan"], row = [], 0
        for s, n in zip(seqs, new):
            first, tokens, pages = pool.pages(s)
            st["plan"].append((row, row + n, first, tokens, torch.from_numpy(pages).to("cuda").long()))
            row += n
    rows = sum(new)
    st["out"] = torch.empty((rows, case["heads"], case["d"]), dtype=DTYPES[case["dtype"]], device="cuda")
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    if case["kind"] == "pages":
        tables, moved = _grow_and_prune(st["pool"], case)
        return {"keys": st["keys"], "values": st["values"], "moved": moved,
                "tables": [t for _, _, t in tables], "tokens": [n for _, n, _ in tables]}
    if case["kind"] == "norm_rope":
        if own:
            st["batch"].qk_norm_rope(0, st["qkv"], st["gq"], st["gk"], st["positions"], THETA, st["out"])
        else:
            _norm_rope(st)
        return {"q": st["out"], "keys": st["keys"], "values": st["values"]}
    if own:
        st["batch"].attention(0, st["q"], st["out"])
    else:
        _attention(st)
    return st["out"]


def _axis_dims(d, axes):
    return [d] if axes == 1 else [d - 4 * (d // 6), 2 * (d // 6), 2 * (d // 6)]


def _norm_rope(st):
    case = st["case"]
    kv, d, heads, page = case["kv_heads"], case["d"], case["heads"], case["page"]
    # the angles in 64 bits: positions go far
    ang = [st["positions"][:, a:a + 1].double() * THETA ** (-torch.arange(0, n, 2, device="cuda").double() / n)
           for a, n in enumerate(_axis_dims(d, case["axes"]))]
    ang = torch.cat(ang, 1)[:, None]
    cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
    q, k, v = st["qkv"].float().view(-1, heads + 2 * kv, d).split((heads, kv, kv), 1)

    def norm_rotate(x, gain):
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)

    st["out"].copy_(norm_rotate(q, st["gq"]))
    k = norm_rotate(k, st["gk"]).to(st["keys"].dtype)
    v = v.to(st["values"].dtype)
    for lo, hi, first, tokens, pages in st["plan"]:
        at = first + tokens - (hi - lo) + torch.arange(hi - lo, device="cuda")
        st["keys"][0, pages[at // page], :, at % page] = k[lo:hi]
        st["values"][0, pages[at // page], :, at % page] = v[lo:hi]


def _attention(st):
    case = st["case"]
    kv, d, page = case["kv_heads"], case["d"], case["page"]
    group = case["heads"] // kv
    scale = 1.0 / math.sqrt(d)
    for lo, hi, first, tokens, pages in st["plan"]:
        # [kv_heads, keys, d]
        k, v = (b[0, pages].permute(1, 0, 2, 3).reshape(kv, -1, d)[:, first:first + tokens].float()
                for b in (st["keys"], st["values"]))
        step = max(1, (1 << 28) // (case["heads"] * tokens))
        for a in range(lo, hi, step):
            b = min(a + step, hi)
            q = st["q"][a:b].float().view(b - a, kv, group, d).permute(1, 0, 2, 3).reshape(kv, -1, d)
            s = torch.matmul(q, k.transpose(1, 2)) * scale
            p = torch.exp(s - s.amax(-1, keepdim=True))
            o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
            st["out"][a:b] = o.view(kv, b - a, group, d).permute(1, 0, 2, 3).reshape(b - a, -1, d)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    if case["kind"] == "pages":
        return None  # nothing is computed: bytes are moved
    x = _inputs(case, seed)
    pool = Pages(x["keys"], x["values"], case["page"], x["keys"].shape[1], case["branches"] + 1)
    seqs, new = _branches(pool, case)
    if case["kind"] == "norm_rope":
        return _exact_norm_rope(case, x, pool, seqs, new)
    heads, kv, d = case["heads"], case["kv_heads"], case["d"]
    out = torch.empty((sum(new), heads, d), dtype=torch.float64, device="cuda")
    row = 0
    for s, n in zip(seqs, new):
        first, tokens, pages = pool.pages(s)
        at = torch.arange(first, first + tokens, device="cuda")
        page_of = torch.from_numpy(pages).to("cuda").long()[at // case["page"]]
        for h in range(heads):
            k = x["keys"][0, page_of, h * kv // heads, at % case["page"]].double()
            v = x["values"][0, page_of, h * kv // heads, at % case["page"]].double()
            for lo in range(0, n, 4096):
                q = x["q"][row + lo:row + min(lo + 4096, n), h].double()
                out[row + lo:row + lo + len(q), h] = torch.softmax(q @ k.T.contiguous() / d ** 0.5, 1) @ v
        row += n
    return out


def _exact_norm_rope(case, x, pool, seqs, new):
    heads, kv, d, page = case["heads"], case["kv_heads"], case["d"], case["page"]
    keys, values = x["keys"].double(), x["values"].double()
    qkv = x["qkv"].double()
    turns = []
    for axis, n in enumerate(_axis_dims(d, case["axes"])):
        for i in range(n // 2):
            turns.append(x["positions"][:, axis].double() * math.exp(-2.0 * i / n * math.log(THETA)))
    turn = torch.polar(torch.ones_like(turns[0])[:, None], torch.stack(turns, 1))

    def head(col, gain):
        y = qkv[:, col * d:(col + 1) * d]
        y = y / (y.square().sum(1, keepdim=True) / d + EPS).sqrt() * gain.double()
        return torch.view_as_real(torch.view_as_complex(y.view(-1, d // 2, 2).contiguous()) * turn).reshape(-1, d)

    q = torch.stack([head(h, x["gq"]) for h in range(heads)], 1)
    k = [head(heads + h, x["gk"]) for h in range(kv)]
    row = 0
    for s, n in zip(seqs, new):
        first, tokens, pages = pool.pages(s)
        for i0 in range(0, n, page):
            i = np.arange(i0, min(i0 + page, n))
            at = first + tokens - n + i
            p, r, rows = (torch.from_numpy(a).cuda().long() for a in (pages[at // page], at % page, row + i))
            for h in range(kv):
                keys[0, p, h, r] = k[h][rows]
                col = (heads + kv + h) * d
                values[0, p, h, r] = qkv[rows, col:col + d]
        row += n
    return {"q": q, "keys": keys, "values": values}
