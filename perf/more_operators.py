"""A prompt's way into the cache and differential attention, as cases to time and compare: each in the framework's kernels and in
elementary torch operations.

  pages     attention of a chunk of new tokens over a paged FP16 cache: every sequence's new keys and values go to its pages,
            every new token attends the sequence's earlier tokens and the chunk's up to itself.  Sequences of different lengths
            together, from a single token to a whole prompt; with `diff` the difference of two softmax maps per pair of heads.
  diff      differential attention of a decode step over the mixed INT8 / FP16 cache, for `layers` layers, its importance, and the
            conf_kv_evict_compact that ends the step.  The budgets and the protected window equal the cache's length, so
            a step drops the oldest tokens and keeps the rest: the cache is a window that slides.
  handover  a prompt that lies in pages becomes the mixed cache, layer by layer, and the first decode step is taken on it.
"""
import math

import torch

own = False


def listed():
    return [
        # One sequence, one token behind a short chat: the smallest call there is.
        _pages("pages_b1", context=1000),
        # A decode step of a full batch, contexts of every length.
        _pages("pages_b32", batch=32, context=8192, page=64, ragged=True, tokens=1),
        # One chunk of a long prompt: chunked prefill behind what came before.
        _pages("pages_chunk_512", tokens=512, context=14987),
        # Four whole prompts: the largest.
        _pages("pages_prompt_4x8192", batch=4, tokens=8192, page=256),
        # Continuous batching: prompts' chunks, single tokens and idle sequences in one call, rows packed.
        _pages("pages_mixed_16", batch=16, tokens=700, context=5000, heads=40, page=32, ragged=True, heads_first=True),
        # A small multi-head model's prompts of odd length.
        _pages("pages_4x333", batch=4, tokens=333, heads=12, kv_heads=12, dim=64),
        # Chunks of a model with differential attention.
        _pages("pages_diff_2x1024", batch=2, tokens=1024, context=4096, page=64, diff=True),
        # One short sequence of a small model, FP16 storage only: latency.
        _diff("diff_b1_512", batch=1, heads=24, kv_heads=12, dim=64, cache=512, window=-1),
        # A batch of long sequences, nearly all INT8.
        _diff("diff_b8_4096", batch=8, cache=4096, layers=4),
        # Draft tokens, four at a time.
        _diff("diff_b16_chunk4", batch=16, tokens=4, cache=1027, window=64, layers=2),
        # A short prompt of a small model.
        _handover("handover_b1_1003", heads=12, kv_heads=12, dim=64, prompt=1003),
        # A batch of long prompts.
        _handover("handover_b8_8192", batch=8, prompt=8192, page=64, heads_first=True, layers=4),
    ]


def _pages(name=None, batch=1, tokens=1, context=0, heads=32, kv_heads=8, dim=128, page=16, ragged=False, heads_first=False,
           diff=False):
    return _named(name, op="pages", batch=batch, tokens=tokens, context=context, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                  ragged=ragged, heads_first=heads_first, diff=diff)


def _diff(name=None, batch=1, tokens=1, heads=32, kv_heads=8, dim=128, cache=512, window=128, layers=1):
    return _named(name, op="diff", batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, cache=cache, window=window,
                  layers=layers)


def _handover(name=None, batch=1, heads=32, kv_heads=8, dim=128, prompt=512, window=128, page=16, heads_first=False, layers=1):
    return _named(name, op="handover", batch=batch, tokens=1, heads=heads, kv_heads=kv_heads, dim=dim, prompt=prompt, window=window,
                  page=page, heads_first=heads_first, layers=layers)


def _named(name, **c):
    return c if name is None else dict(c, name=name)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: batches of 1 to 32, chunks of 1 to 8192 tokens behind up to 32768, caches and prompts of 130 to 8192, 1 to 16
    query heads per kv-head."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    op = rng.choice(["pages", "pages", "diff", "handover"])
    while True:
        dim, kv, batch = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 12]), _log_int(rng, 1, 32)
        group = rng.choice([1, 2, 4, 4, 5, 6, 7, 8] + ([12, 16] if dim == 128 else []))
        if op == "pages":
            diff = group % 2 == 0 and rng.random() < 0.3
            c = _pages(batch=batch, tokens=rng.choice([1, _log_int(rng, 1, 16), _log_int(rng, 2, 8192)]),
                       context=rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 1, 32768)]), heads=kv * group, kv_heads=kv, dim=dim,
                       page=rng.choice([8, 16, 16, 32, 64, 128, 256, 1024]), ragged=rng.random() < 0.5,
                       heads_first=rng.random() < 0.5, diff=diff)
        elif op == "diff":
            if group % 2:
                continue
            c = _diff(batch=batch, tokens=rng.choice([1, 1, 1, 2, 4]), heads=kv * group, kv_heads=kv, dim=dim,
                      cache=_log_int(rng, 130, 8192), window=rng.choice([-1, 32, 64, 128]), layers=rng.choice([1, 2, 4]))
            if c["tokens"] > 1 and (dim != 128 or c["tokens"] * group > 16):
                continue
        else:
            c = _handover(batch=batch, heads=kv * group, kv_heads=kv, dim=dim, prompt=_log_int(rng, 130, 8192),
                          window=rng.choice([-1, 32, 64, 128]), page=rng.choice([8, 16, 16, 32, 64, 128, 256]),
                          heads_first=rng.random() < 0.5, layers=rng.choice([1, 2, 4]))
        if _cost(c) <= most[op] and work(c)["bytes"] <= 2e9:
            return c


def _lengths(c):
    """(new tokens, tokens before them) of every sequence of a call: all alike, or with `ragged` chunks of several lengths, single
    tokens and sequences that sit the call out."""
    T, C, new, context = c["tokens"], c["context"], [], []
    for b in range(c["batch"]):
        if not c["ragged"]:
            new.append(T)
            context.append(C)
        else:
            new.append((T, 1, -(-T // 3), 0, min(2, T))[b % 5])
            context.append((C * (b + 1) // c["batch"], C, C // 7, C // 2, 0, max(C - 1, 0), C // 3)[b % 7])
    return new, context


def work(c):
    """Bytes and operations of one pass: every input read once, every output written once (a cache's stored rows and scales,
    its importance read and written), two operations per multiply-add of the two contractions."""
    Hq, H, D, B = c["heads"], c["kv_heads"], c["dim"], c["batch"]
    if c["op"] == "pages":
        new, context = _lengths(c)
        rows = float(sum(new))
        kept = float(sum(n0 for n, n0 in zip(new, context) if n))
        pairs = float(sum(n * n0 + n * (n + 1) // 2 for n, n0 in zip(new, context)))
        outs = Hq // 2 if c["diff"] else Hq
        extra = 4.0 * outs * rows if c["diff"] else 0.0
        return {"bytes": kept * H * 4 * D + rows * H * 8 * D + rows * (Hq + outs) * 2 * D + extra, "flops": 4.0 * D * Hq * pairs}
    if c["op"] == "handover":
        N = c["prompt"]
        n16 = N if c["window"] < 0 else min(N, c["window"])
        stored = (N - n16) * (2 * D + 4) + n16 * 4 * D + 8.0 * N
        row = N * 4.0 * D + stored + 8 * D + 12
        return {"bytes": c["layers"] * B * (H * row + Hq * 4.0 * D), "flops": c["layers"] * 4.0 * B * Hq * (N + 1) * D}
    N, tq = c["cache"], c["tokens"]
    n16 = N if c["window"] < 0 else min(N, c["window"])
    row = (N - n16) * (2 * D + 4) + n16 * 4 * D + 8.0 * (N + tq) + tq * 8 * D
    per_layer = B * H * row + B * tq * Hq * (3.0 * D + 2)
    return {"bytes": c["layers"] * per_layer, "flops": c["layers"] * 4.0 * B * tq * Hq * (N + tq) * D}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 200)


# ---- inputs ----

class _State:
    pass


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 31)
    return g


class _Values:
    """Normal values, and queries and keys of one kv-head that lean the same way (some keys: those a query looks for)."""

    def __init__(self, c, seed):
        self.c, self.g = c, _generator(seed)
        self.u = torch.nn.functional.normalize(self.normal(c["kv_heads"], c["dim"]).float(), dim=-1)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float16)

    def queries(self, *shape):
        """[..][Hq][D]; the two maps of a pair differ."""
        Hq, H, D = self.c["heads"], self.c["kv_heads"], self.c["dim"]
        mean = (math.sqrt(D) * self.u).repeat_interleave(Hq // H, dim=0)
        return self.normal(*shape, Hq, D).add_(mean.half())

    def keys(self, *shape):
        """[..][Hkv][D]."""
        k = self.normal(*shape, *self.u.shape)
        lean = torch.rand(*shape, len(self.u), 1, generator=self.g, device="cuda") < 0.02
        return k.add_(lean * (3.0 * self.u).half())

    def weights(self, *shape):
        """Learned weights of the second map."""
        return 0.2 + 0.7 * torch.rand(*shape, self.c["heads"] // 2, generator=self.g, device="cuda")


def _room(c, sequences, seed_of):
    """Pages for sequences of these lengths, handed out in no order, and the table that finds them (entries behind a sequence's end:
    -1)."""
    page = c["page"]
    counts = [-(-n // page) for n in sequences]
    total, most = max(1, sum(counts)), max(1, max(counts))
    order = torch.randperm(total, generator=seed_of, device="cuda").int()
    table, at = torch.full((len(sequences), most), -1, dtype=torch.int32, device="cuda"), 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at:at + n]
        at += n
    return total, table


def _paged(c, planes):
    """[pages][page][Hkv][D] as the program sees it; in memory the heads of a token may lie apart."""
    return planes.transpose(1, 2).contiguous().transpose(1, 2) if c["heads_first"] else planes


def _pages_inputs(c, seed):
    x, st = _Values(c, seed), _State()
    H, D = c["kv_heads"], c["dim"]
    st.new, st.context = _lengths(c)
    n, st.table = _room(c, [a + b for a, b in zip(st.new, st.context)], x.g)
    st.pages_k, st.pages_v = _paged(c, x.keys(n, c["page"])), _paged(c, x.normal(n, c["page"], H, D))
    st.starts = [sum(st.new[:b]) for b in range(c["batch"])]
    R = max(1, sum(st.new))
    st.q, st.k, st.v = x.queries(R), x.keys(R), x.normal(R, H, D)
    st.lam = x.weights(R) if c["diff"] else None
    return st


def _diff_inputs(c, seed):
    x, st = _Values(c, seed), _State()
    L, B, tq, H, D, N = (c[k] for k in ("layers", "batch", "tokens", "kv_heads", "dim", "cache"))
    st.q, st.k, st.v = x.queries(L, B, tq), x.keys(L, B, tq), x.normal(L, B, tq, H, D)
    st.cache_k, st.cache_v = x.keys(L, B, N).transpose(2, 3).contiguous(), x.normal(L, B, H, N, D)
    st.lam = x.weights(L, B, tq)
    return st


def _handover_inputs(c, seed):
    x, st = _Values(c, seed), _State()
    L, B, H, D = (c[k] for k in ("layers", "batch", "kv_heads", "dim"))
    n, st.table = _room(c, [c["prompt"]] * B, x.g)
    st.pages = [(_paged(c, x.keys(n, c["page"])), _paged(c, x.normal(n, c["page"], H, D))) for _ in range(L)]
    st.q, st.k, st.v = x.queries(L, B), x.keys(L, B), x.normal(L, B, H, D)
    return st


def _handle(c, **kw):
    """The cache manager that a serving program keeps."""
    from paper_2605_24786_amd import ConfKV
    shape = dict(n_layers=1, batch=c["batch"], n_q_heads=c["heads"], n_kv_heads=c["kv_heads"], head_dim=c["dim"], vocab=32000,
                 capacity=64, fp16_window=16, protected_window=16, n_tight=[32], n_loose=[32])
    return ConfKV(**dict(shape, **kw))


def prepare(c, seed):
    if c["op"] == "pages":
        st = _pages_inputs(c, seed)
        if own:
            i32 = dict(dtype=torch.int32, device="cuda")
            st.kv = _handle(c, max_paged=st.table.shape[1] * c["page"])
            st.out = torch.empty(len(st.q), c["heads"] // 2 if c["diff"] else c["heads"], c["dim"], dtype=torch.float16, device="cuda")
            st.at, st.count, st.before = (torch.tensor(x, **i32) for x in (st.starts, st.new, st.context))
    elif c["op"] == "diff":
        st = _diff_inputs(c, seed)
        L, B, N, tq, Hq, D = (c[k] for k in ("layers", "batch", "cache", "tokens", "heads", "dim"))
        if own:
            st.kv = _handle(c, n_layers=L, capacity=-(-(N + tq) // 64) * 64, fp16_window=c["window"], protected_window=N,
                            n_tight=[N] * L, n_loose=[N] * L, max_chunk=tq if tq > 1 else 0)
            for l in range(L):
                st.kv.load_prefill(l, st.cache_k[l], st.cache_v[l])
            st.out = torch.empty(L, B, tq, Hq // 2, D, dtype=torch.float16, device="cuda")
        else:
            st.rows = [[_stored(c, x[l].float()) for x in (st.cache_k, st.cache_v)] for l in range(L)]
            st.mass = [torch.zeros(st.cache_k.shape[1:4], device="cuda") for _ in range(L)]
    else:
        st = _handover_inputs(c, seed)
        L, N = c["layers"], c["prompt"]
        if own:
            st.kv = _handle(c, n_layers=L, capacity=-(-(N + 1) // 64) * 64, fp16_window=c["window"], protected_window=N,
                            n_tight=[N] * L, n_loose=[N] * L)
            st.out = torch.empty_like(st.q)
    st.case = c
    return st


def run(st):
    return {"pages": _run_pages, "diff": _run_diff, "handover": _run_handover}[st.case["op"]](st)


# ---- a chunk over pages ----

def _run_pages(st):
    c = st.case
    if own:
        st.kv.attend_pages(st.q, st.k, st.v, st.out, st.pages_k, st.pages_v, st.table, st.before, tokens=c["tokens"], starts=st.at,
                           new=st.count, lam=st.lam)
        return {"out": st.out[:sum(st.new)], "k": st.pages_k, "v": st.pages_v}
    Hq, H, D, page, dev = c["heads"], c["kv_heads"], c["dim"], c["page"], st.q.device
    G = Hq // H
    outs = []
    for b, (n, n0, s) in enumerate(zip(st.new, st.context, st.starts)):
        if n == 0:
            continue
        at = torch.arange(n0 + n, device=dev)
        pages, slots = st.table[b, at // page].long(), at % page
        for plane, rows in ((st.pages_k, st.k), (st.pages_v, st.v)):
            plane[pages[n0:], slots[n0:]] = rows[s:s + n]
        k, v = (plane[pages, slots].float().transpose(0, 1) for plane in (st.pages_k, st.pages_v))         # [H][n0 + n][D]
        q = st.q[s:s + n].float().reshape(n, H, G, D).permute(1, 2, 0, 3).reshape(H, G * n, D)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).reshape(H, G, n, n0 + n) / math.sqrt(D)
        x.masked_fill_(at > n0 + torch.arange(n, device=dev)[:, None], -math.inf)
        x = (x - x.amax(-1, keepdim=True)).exp_()
        x /= x.sum(-1, keepdim=True)
        if st.lam is not None:
            lam = st.lam[s:s + n].reshape(n, H, G // 2).permute(1, 2, 0)[..., None]
            x = x[:, 0::2] - lam * x[:, 1::2]
        o = torch.matmul(x.reshape(H, -1, n0 + n), v).reshape(H, -1, n, D).permute(2, 0, 1, 3)
        outs.append(o.reshape(n, -1, D).half())
    return {"out": torch.cat(outs) if outs else st.q[:0], "k": st.pages_k, "v": st.pages_v}


# ---- the mixed cache ----

def _codes(x):
    """Rows x as INT8 storage keeps them: codes times one FP16 scale per row, largest magnitude / 127.  (The quotient in 64
    bits: it decides between two codes.)"""
    s = (x.abs().amax(-1, keepdim=True) / 127.0).half().float()
    codes = (x.double() / torch.where(s > 0, s, 1.0).double()).round().clamp(-127, 127).float()
    return torch.where(s > 0, codes * s, 0.0)


def _stored(c, x):
    """A cache's rows [B][H][N][D]: all but the newest `window` tokens as INT8."""
    old = 0 if c["window"] < 0 else max(0, x.shape[2] - c["window"])
    return torch.cat([_codes(x[:, :, :old]), x[:, :, old:]], 2)


def _maps(c, q, k):
    """Probabilities [B][H][tq][G][N] of queries [B][tq][Hq][D] over rows k [B][H][N][D], the last tq of them the call's own."""
    B, tq, Hq, D = q.shape
    H, n = k.shape[1:3]
    G = Hq // H
    q = q.float().reshape(B, tq, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, tq * G, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).reshape(B, H, tq, G, n) / math.sqrt(D)
    later = torch.arange(n, device=q.device) > n - tq + torch.arange(tq, device=q.device)[:, None]
    x = x.masked_fill(later[:, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    return p / p.sum(-1, keepdim=True)


def _weighted(p, v):
    """Weights [B][H][tq][J][N] of rows v [B][H][N][D] -> [B][tq][H * J][D]."""
    B, H, tq, J, n = p.shape
    o = torch.matmul(p.reshape(B, H, tq * J, n), v).reshape(B, H, tq, J, -1)
    return o.permute(0, 2, 1, 3, 4).reshape(B, tq, H * J, -1).half()


# ---- differential attention over it ----

def _run_diff(st):
    c = st.case
    if own:
        for l in range(c["layers"]):
            st.kv.attend_diff(l, st.q[l], st.k[l], st.v[l], st.out[l], st.lam[l])
        st.kv.evict_compact()
        return st.out
    return torch.stack([_layer(c, st, l) for l in range(c["layers"])])


def _layer(c, st, l):
    B, tq, H, N, W = (c[k] for k in ("batch", "tokens", "kv_heads", "cache", "window"))
    k, v = (torch.cat([old, new[l].transpose(1, 2).float()], 2) for old, new in zip(st.rows[l], (st.k, st.v)))
    p = _maps(c, st.q[l], k)
    lam = st.lam[l].reshape(B, tq, H, -1).transpose(1, 2)[..., None]
    p = p[:, :, :, 0::2] - lam * p[:, :, :, 1::2]
    out = _weighted(p, v)
    weight, mass = p.abs().sum(3), torch.cat([st.mass[l], torch.zeros(B, H, tq, device="cuda")], 2)
    for t in range(tq):
        mass = 0.9 * mass + 0.1 * weight[:, :, t]
    st.mass[l], moved = mass[:, :, tq:], []
    for x in (k, v):
        x = x[:, :, tq:]
        if 0 <= W < N:
            lo = max(0, N - W - tq)
            x = torch.cat([x[:, :, :lo], _codes(x[:, :, lo:N - W]), x[:, :, N - W:]], 2)
        moved.append(x)
    st.rows[l] = moved
    return out


# ---- a paged prompt becomes the cache ----

def _run_handover(st):
    c = st.case
    N, page = c["prompt"], c["page"]
    if own:
        for l in range(c["layers"]):
            st.kv.load_pages(l, *st.pages[l], st.table, N)
            st.kv.attend(l, st.q[l], st.k[l], st.v[l], st.out[l])
        st.kv.evict_compact()
        return st.out
    at = torch.arange(N, device="cuda")
    pages, slots = st.table[:, at // page].long(), at % page                      # [B][N]
    outs = []
    for l in range(c["layers"]):
        k, v = (torch.cat([_stored(c, plane[pages, slots].transpose(1, 2).float()), new[l].float()[:, :, None]], 2)
                for plane, new in zip(st.pages[l], (st.k, st.v)))
        outs.append(_weighted(_maps(c, st.q[l][:, None], k), v)[:, 0])
    return torch.stack(outs)


# ---- the same in 64 bits ----

def exact(c, seed):
    return {"pages": _exact_pages, "diff": _exact_diff, "handover": _exact_handover}[c["op"]](c, seed)


def _head(q, k, v, first, scale, lam=None):
    """Queries [t][G][D] of one kv-head over rows k, v [n][D]; query t sees the first `first` + t + 1 of them.  A query block at a
    time; with lam [t][G / 2] heads are subtracted in pairs."""
    t, G, D = q.shape
    outs = []
    step = max(1, (1 << 25) // (G * len(k)))
    for lo in range(0, t, step):
        hi = min(t, lo + step)
        n = min(len(k), first + hi)
        s = (q[lo:hi].double().reshape(-1, D) @ k[:n].double().T.contiguous()).reshape(hi - lo, G, n) * scale
        last = first + torch.arange(lo, hi, device=s.device)
        s = s.masked_fill(torch.arange(n, device=s.device) > last[:, None, None], -math.inf)
        o = (torch.softmax(s, -1).reshape(-1, n) @ v[:n].double()).reshape(hi - lo, G, D)
        outs.append(o if lam is None else o[:, 0::2] - lam[lo:hi, :, None].double() * o[:, 1::2])
    return torch.cat(outs)


def _scale(c):
    return float(torch.tensor(1.0 / math.sqrt(c["dim"])))


def _exact_pages(c, seed):
    """Sequence by sequence and head by head, its tokens laid end to end page by page."""
    st = _pages_inputs(c, seed)
    H, G, page = c["kv_heads"], c["heads"] // c["kv_heads"], c["page"]
    outs = []
    for b, (n, n0, s) in enumerate(zip(st.new, st.context, st.starts)):
        if n == 0:
            continue
        ids = st.table[b].tolist()[:-(-(n0 + n) // page)]
        rows = []
        for plane, new in ((st.pages_k, st.k), (st.pages_v, st.v)):
            whole = torch.cat([torch.cat([plane[i] for i in ids])[:n0], new[s:s + n]])
            for j, i in enumerate(ids):
                part = whole[j * page:(j + 1) * page]
                plane[i][:len(part)] = part
            rows.append(whole)
        heads = []
        for h in range(H):
            lam = None if st.lam is None else st.lam[s:s + n, h * G // 2:(h + 1) * G // 2]
            heads.append(_head(st.q[s:s + n, h * G:(h + 1) * G], rows[0][:, h], rows[1][:, h], n0, _scale(c), lam))
        outs.append(torch.cat(heads, 1))
    out = torch.cat(outs) if outs else st.q[:0].double()
    return {"out": out, "k": st.pages_k, "v": st.pages_v}


def _mixed(c, x):
    """Rows [n][D] of one sequence and head in 64 bits, all but the newest `window` through the INT8 codes."""
    x, W = x.double(), c["window"]
    if 0 <= W < len(x):
        x = x.clone()
        o = x[:len(x) - W]
        s = (o.abs().amax(-1, keepdim=True).float() / 127.0).half().double()
        x[:len(x) - W] = torch.where(s > 0, (o / s.clamp(min=1e-300)).round().clamp(-127, 127) * s, 0.0)
    return x


def _exact_diff(c, seed):
    st = _diff_inputs(c, seed)
    L, B, tq, H, N = (c[k] for k in ("layers", "batch", "tokens", "kv_heads", "cache"))
    G = c["heads"] // H
    out = torch.empty(L, B, tq, c["heads"] // 2, c["dim"], dtype=torch.float64, device="cuda")
    for l in range(L):
        for b in range(B):
            for h in range(H):
                k, v = (torch.cat([_mixed(c, old[l, b, h]), new[l, b, :, h].double()])
                        for old, new in ((st.cache_k, st.k), (st.cache_v, st.v)))
                pairs = slice(h * G // 2, (h + 1) * G // 2)
                out[l, b, :, pairs] = _head(st.q[l, b, :, h * G:(h + 1) * G], k, v, N, _scale(c), st.lam[l, b, :, pairs])
    return out


def _exact_handover(c, seed):
    st = _handover_inputs(c, seed)
    L, B, H, N, page = (c[k] for k in ("layers", "batch", "kv_heads", "prompt", "page"))
    G = c["heads"] // H
    out = torch.empty(st.q.shape, dtype=torch.float64, device="cuda")
    tables = [row[:-(-N // page)] for row in st.table.tolist()]
    for l in range(L):
        for b in range(B):
            k, v = (torch.cat([plane[i] for i in tables[b]])[:N] for plane in st.pages[l])
            for h in range(H):
                keys, values = (torch.cat([_mixed(c, x[:, h]), new[l, b, h].double()[None]]) for x, new in ((k, st.k), (v, st.v)))
                out[l, b, h * G:(h + 1) * G] = _head(st.q[l, b, None, h * G:(h + 1) * G], keys, values, N, _scale(c))[0]
    return out
