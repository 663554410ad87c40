"""The calls around a decode step's attention, as cases to time and compare: each in the framework's kernels and in
elementary torch operations.

  prepare   queries, keys and values as a projection leaves them become what the cache manager takes: RMS norm of every
            query and key head, position rotation, FP16, the layout of conf_kv_attend(_chunk) or of conf_kv_load_prefill.
  shared    decode attention of a batch whose sequences share a long prefix: softmax over the prefix, which is stored once,
            and the sequence's own cache (mixed INT8 / FP16), for `layers` layers, and the conf_kv_evict_compact that ends
            the step.  The budgets and the protected window equal the cache's length, so a step drops the oldest tokens and
            keeps the rest: the cache is a window that slides.
  constrain logits become what conf_kv_step takes: penalties for repeated tokens, biases, grammar masks, float32.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"fp32": 4, "fp16": 2, "bf16": 2}


def listed():
    return [
        # One sequence, one token: the smallest call there is, a projection's row of 48 heads.
        _prepare("prepare_b1", tokens=1, far=1000, type="bf16"),
        # A decode step of a full batch of a model with five query heads per kv-head and normalised heads.
        _prepare("prepare_b32_norm", batch=32, tokens=1, heads=40, norm=True, type="bf16", far=4096),
        # Eight prompts of 4096 tokens, handed to the cache in its prompt layout.
        _prepare("prepare_prompt_8x4096", batch=8, tokens=4096, norm=True, prompt=True, type="bf16"),
        # A small multi-head model in float32 that rotates half of its 64 channels, neighbours paired; a ragged prompt.
        _prepare("prepare_prompt_1003_half", tokens=1003, heads=12, kv_heads=12, dim=64, rotated=32, paired=True, prompt=True,
                 type="fp32"),
        # Four sequences of a small multi-head model behind a system prompt: latency.
        _shared("shared_b4_512", batch=4, heads=12, kv_heads=12, dim=64, prefix=512, cache=256, window=-1),
        # A small batch behind a long system prompt.
        _shared("shared_b8_8192", batch=8, prefix=8192, cache=1024, layers=4),
        # A full batch, 128 query rows per kv-head against every shared key.
        _shared("shared_b32_4096", batch=32, prefix=4096, cache=512, layers=4),
        # One document, many questions: a ragged prefix that some sequences see in part or not at all.
        _shared("shared_b16_32001", batch=16, heads=40, prefix=32001, cache=700, window=64, ragged=True, layers=2),
        # Draft tokens, four at a time.
        _shared("shared_b8_chunk4", batch=8, tokens=4, prefix=2048, cache=1024, layers=2),
        # One sequence of a small vocabulary, a chat's worth of history.
        _constrain("constrain_b1", vocab=50257, history=300, type="fp32"),
        # A small batch under a grammar, with biases.
        _constrain("constrain_b8_grammar", batch=8, vocab=128256, history=4096, mask=True, bias=300, type="bf16"),
        # A full batch with long histories.
        _constrain("constrain_b32_32k", batch=32, vocab=152064, history=32768, mask=True, bias=64, type="bf16"),
    ]


def _prepare(name=None, batch=1, tokens=1, heads=32, kv_heads=8, dim=128, rotated=0, paired=False, norm=False, prompt=False,
             far=0, type="bf16"):
    return _named(name, op="prepare", batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim,
                  rotated=rotated or dim, paired=paired, norm=norm, prompt=prompt, far=far, type=type)


def _shared(name=None, batch=8, tokens=1, heads=32, kv_heads=8, dim=128, prefix=2048, cache=512, window=128, ragged=False,
            layers=1):
    return _named(name, op="shared", batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, prefix=prefix,
                  cache=cache, window=window, ragged=ragged, layers=layers)


def _constrain(name=None, batch=1, vocab=32000, history=0, bias=0, mask=False, type="fp32"):
    return _named(name, op="constrain", batch=batch, vocab=vocab, history=history, bias=bias, mask=mask, type=type)


def _named(name, **c):
    return c if name is None else dict(c, name=name)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: batches of 1 to 32, prompts and prefixes of up to 32768 tokens, 1 to 16 query heads per kv-head."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    op = rng.choice(["prepare", "shared", "constrain"])
    while True:
        if op == "prepare":
            dim, kv = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 12])
            prompt = rng.random() < 0.5
            c = _prepare(batch=_log_int(rng, 1, 32), tokens=_log_int(rng, 2, 16384) if prompt else rng.choice([1, 1, 1, 3, 4]),
                         heads=kv * rng.choice([1, 2, 4, 5, 7, 8] + ([12, 16] if dim == 128 else [])), kv_heads=kv, dim=dim,
                         rotated=16 * rng.randint(1, dim // 16), paired=rng.random() < 0.3, norm=rng.random() < 0.5,
                         prompt=prompt, far=rng.choice([100, 5000, 1000000]), type=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
        elif op == "shared":
            dim, kv = rng.choice([64, 128, 128, 128]), rng.choice([2, 4, 8, 8, 12])
            group = rng.choice([1, 2, 4, 4, 5, 7, 8] + ([12, 16] if dim == 128 else []))
            window, cache = rng.choice([-1, 32, 64, 128]), _log_int(rng, 130, 4096)
            c = _shared(batch=_log_int(rng, 1, 32), tokens=rng.choice([1, 1, 1, 2, 4]), heads=kv * group, kv_heads=kv, dim=dim,
                        prefix=_log_int(rng, 16, 32768), cache=cache, window=window, ragged=rng.random() < 0.4,
                        layers=rng.choice([1, 2, 4]))
            if c["tokens"] > 1 and (dim != 128 or c["tokens"] * group > 16):
                continue
        else:
            c = _constrain(batch=_log_int(rng, 1, 32), vocab=rng.choice([32000, 50257, 128256, 152064, _log_int(rng, 1000, 152064)]),
                           history=rng.choice([0, _log_int(rng, 1, 32768)]), bias=rng.choice([0, 1, _log_int(rng, 2, 1000)]),
                           mask=rng.random() < 0.6, type=rng.choice(["fp32", "bf16", "fp16"]))
        if _cost(c) <= most[op]:
            return c


def work(c):
    """Bytes and operations of one pass: every input read once, every output written once (a cache's stored rows and scales,
    its importance read and written), two operations per multiply-add of the two contractions."""
    if c["op"] == "prepare":
        values = float(c["batch"] * c["tokens"] * (c["heads"] + 2 * c["kv_heads"]) * c["dim"])
        turned = float(c["batch"] * c["tokens"] * (c["heads"] + c["kv_heads"]) * c["dim"])
        return {"bytes": values * (SIZES[c["type"]] + 2), "flops": turned * (7 if c["norm"] else 3)}
    if c["op"] == "constrain":
        words = -(-c["vocab"] // 32) * 4 if c["mask"] else 0
        row = c["vocab"] * (SIZES[c["type"]] + 4.0) + words + 4.0 * c["history"] + 8.0 * c["bias"]
        return {"bytes": c["batch"] * row, "flops": float(c["batch"] * (c["vocab"] + 6 * c["history"]))}
    B, tq, Hq, H, D, N = (c[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim", "cache"))
    n16 = N if c["window"] < 0 else min(N, c["window"])
    row = (N - n16) * (2 * D + 4) + n16 * 4 * D + 8.0 * (N + tq) + tq * 8 * D
    seen = sum(_seen(c)) / B
    per_layer = H * max(_seen(c)) * 4.0 * D + B * H * row + B * tq * Hq * 4.0 * D
    return {"bytes": c["layers"] * per_layer, "flops": c["layers"] * 4.0 * B * tq * Hq * (seen + N + tq) * D}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _seen(c):
    """Tokens of the prefix that each sequence sees: all, or with `ragged` all, some or none."""
    T = c["prefix"]
    return [(T, (T * (b + 1)) // (c["batch"] + 1), 0, T - 1, T)[b % 5] if c["ragged"] else T for b in range(c["batch"])]


# ---- inputs ----

class _State:
    pass


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + 29)
    return g


def _frequencies(c):
    """Rotation angles per position: 10000^(-2 i / rotated)."""
    i = torch.arange(c["rotated"] // 2, dtype=torch.float64, device="cuda")
    return (10000.0 ** (-2.0 * i / c["rotated"])).float()


def _prepare_inputs(c, seed):
    g, st = _generator(seed), _State()
    B, T, Hq, H, D = (c[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim"))
    rows = torch.randn(B, T, Hq + 2 * H, D, generator=g, device="cuda", dtype=TYPES[c["type"]])
    rows *= 1.0 + 2.0 * torch.rand(Hq + 2 * H, 1, generator=g, device="cuda").to(rows.dtype)      # heads differ in size
    st.q, st.k, st.v = rows[:, :, :Hq], rows[:, :, Hq:Hq + H], rows[:, :, Hq + H:]
    st.wq = st.wk = None
    if c["norm"]:
        st.wq, st.wk = (1.0 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
    st.freq = _frequencies(c)
    # a sequence starts anywhere below `far`; its tokens follow one another
    start = torch.randint(0, c["far"] + 1, (B, 1), generator=g, device="cuda", dtype=torch.int32)
    st.pos = start + torch.arange(T, device="cuda", dtype=torch.int32)
    return st


def _shared_inputs(c, seed):
    g, st = _generator(seed), _State()
    L, B, tq, Hq, H, D, T, N = (c[k] for k in ("layers", "batch", "tokens", "heads", "kv_heads", "dim", "prefix", "cache"))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)

    def keys(*shape):
        """Keys of which a few lean towards the queries of their head (dimension 1)."""
        k = normal(*shape, D)
        lean = torch.rand(shape, generator=g, device="cuda") < 0.02
        return k.add_(lean[..., None] * (3.0 * u[:, :, None] if len(shape) == 3 else 3.0 * u[:, None, :, None]).to(k.dtype))

    u = torch.nn.functional.normalize(normal(L, H, D).float(), dim=-1)
    mean = (math.sqrt(D) * u).repeat_interleave(Hq // H, dim=1).half()
    st.q = normal(L, B, tq, Hq, D).add_(mean[:, None, None])
    st.k, st.v = normal(L, B, tq, H, D), normal(L, B, tq, H, D)
    st.shared_k, st.shared_v = keys(L, H, T), normal(L, H, T, D)
    st.cache_k, st.cache_v = keys(L, B, H, N), normal(L, B, H, N, D)
    st.seen = torch.tensor(_seen(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
    return st


def _constrain_inputs(c, seed):
    g, st = _generator(seed), _State()
    B, V, n, m = c["batch"], c["vocab"], c["history"], c["bias"]

    def uniform(lo, hi):
        return lo + (hi - lo) * torch.rand(B, generator=g, device="cuda")

    st.logits = (3.0 * torch.randn(B, V, generator=g, device="cuda")).to(TYPES[c["type"]])
    # text repeats itself: a token's rank falls off like a power
    st.tokens = (V ** torch.rand(B, max(n, 1), generator=g, device="cuda")).int().clamp(max=V - 1) - 1
    st.tokens.clamp_(min=0)
    st.lengths = (n * (1.0 - 0.3 * torch.rand(B, generator=g, device="cuda"))).int()
    st.prompt_lengths = st.lengths // 2
    st.repetition, st.presence, st.frequency = uniform(1.0, 1.5), uniform(-0.5, 1.0), uniform(0.0, 0.2)
    st.bias_offsets = m * torch.arange(B + 1, dtype=torch.int32, device="cuda")
    st.bias_tokens = torch.randint(0, V, (B * m,), generator=g, device="cuda", dtype=torch.int32)
    if m:                                          # no token twice: a row's tokens are spread evenly from a start of its own
        first = torch.randint(0, V, (B, 1), generator=g, device="cuda")
        st.bias_tokens = ((first + torch.arange(m, device="cuda") * max(1, V // m)) % V).int().reshape(-1)
    st.bias_values = 4.0 * torch.randn(B * m, generator=g, device="cuda")
    st.bias_values[::5] = -math.inf                # banned tokens among them
    words = -(-V // 32)
    # grammars allow anything from nearly all tokens to a handful
    share = torch.rand(B, 1, generator=g, device="cuda") ** 3
    bits = torch.rand(B, words * 32, generator=g, device="cuda") < share
    st.bits = bits if c["mask"] else None
    weights = (1 << torch.arange(32, dtype=torch.int64, device="cuda"))
    packed = (bits.reshape(B, words, 32).long() * weights).sum(-1)
    st.allowed = (packed - ((packed >> 31) << 32)).int() if c["mask"] else None
    return st


def _handle(c, **kw):
    """The cache manager that a serving program keeps."""
    from paper_2605_24786_amd import ConfKV
    shape = dict(n_layers=1, batch=c["batch"], n_q_heads=c.get("heads", 1), n_kv_heads=c.get("kv_heads", 1),
                 head_dim=c.get("dim", 128), vocab=c.get("vocab", 32000), capacity=64, fp16_window=16, protected_window=16,
                 n_tight=[32], n_loose=[32])
    return ConfKV(**dict(shape, **kw))


def prepare(c, seed):
    if c["op"] == "prepare":
        st = _prepare_inputs(c, seed)
        B, T, Hq, H, D = (c[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim"))
        if own:
            st.kv = _handle(c)
            st.q16 = torch.empty(B, T, Hq, D, dtype=torch.float16, device="cuda")
            rows = (B, H, T, D) if c["prompt"] else (B, T, H, D)
            st.k16, st.v16 = (torch.empty(rows, dtype=torch.float16, device="cuda") for _ in range(2))
    elif c["op"] == "constrain":
        st = _constrain_inputs(c, seed)
        if own:
            st.kv = _handle(c)
            st.out = torch.empty(c["batch"], c["vocab"], device="cuda")
    else:
        st = _shared_inputs(c, seed)
        L, N, tq = c["layers"], c["cache"], c["tokens"]
        if own:
            st.kv = _handle(c, n_layers=L, capacity=-(-(N + tq) // 64) * 64, fp16_window=c["window"], protected_window=N,
                            n_tight=[N] * L, n_loose=[N] * L, max_chunk=tq if tq > 1 else 0, max_shared=c["prefix"])
            for l in range(L):
                st.kv.load_prefill(l, st.cache_k[l], st.cache_v[l])
            st.out = torch.empty_like(st.q)
        else:
            st.rows = [[_stored(c, x[l].float()) for x in (st.cache_k, st.cache_v)] for l in range(L)]
    st.case = c
    return st


def run(st):
    return {"prepare": _run_prepare, "shared": _run_shared, "constrain": _run_constrain}[st.case["op"]](st)


# ---- queries, keys and values ----

EPS = 1e-6


def _run_prepare(st):
    c = st.case
    if own:
        st.kv.prepare_qkv(0, st.q, st.k, st.v, st.q16, st.k16, st.v16, freq=st.freq, pos=st.pos, q_weight=st.wq,
                          k_weight=st.wk, eps=EPS, interleaved=c["paired"], prompt=c["prompt"])
        return {"q": st.q16, "k": st.k16, "v": st.v16}
    angle = st.pos.double()[..., None] * st.freq.double()                # [B][T][rotated / 2]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    q, k = (_turned(c, _normed(x.float(), w), cos, sin) for x, w in ((st.q, st.wq), (st.k, st.wk)))
    v = st.v
    if c["prompt"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return {"q": q.half(), "k": k.half().contiguous(), "v": v.float().half().contiguous()}


def _normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _turned(c, x, cos, sin):
    R = c["rotated"]
    if c["paired"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., R:]], -1)


# ---- attention over a shared prefix and the sequence's cache ----

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


def _run_shared(st):
    c = st.case
    if own:
        for l in range(c["layers"]):
            st.kv.attend_shared(l, st.q[l], st.k[l], st.v[l], st.out[l], st.shared_k[l], st.shared_v[l], seen=st.seen)
        st.kv.evict_compact()
        return st.out
    return torch.stack([_layer(c, st, l) for l in range(c["layers"])])


def _layer(c, st, l):
    """Scores against the prefix and the cache, one softmax over both, and the window moved on by the call's tokens."""
    B, tq, Hq, H, D, T, N = (c[k] for k in ("batch", "tokens", "heads", "kv_heads", "dim", "prefix", "cache"))
    G, dev = Hq // H, st.q.device
    k, v = (torch.cat([old, new[l].transpose(1, 2).float()], 2) for old, new in zip(st.rows[l], (st.k, st.v)))
    q = st.q[l].float().reshape(B, tq, H, G, D).permute(2, 0, 1, 3, 4)           # [H][B][tq][G][D]
    before = torch.matmul(q.reshape(H, B * tq * G, D), st.shared_k[l].float().transpose(1, 2)).reshape(H, B, tq, G, T)
    if st.seen is not None:
        hidden = torch.arange(T, device=dev) >= st.seen[:, None]
        before = before.masked_fill(hidden[None, :, None, None], -math.inf)
    mine = torch.matmul(q.permute(1, 0, 2, 3, 4).reshape(B, H, tq * G, D), k.transpose(2, 3)).reshape(B, H, tq, G, N + tq)
    later = torch.arange(N + tq, device=dev) > N + torch.arange(tq, device=dev)[:, None]
    mine = mine.masked_fill(later[:, None], -math.inf).permute(1, 0, 2, 3, 4)
    s = torch.cat([before, mine], -1) / math.sqrt(D)
    p = (s - s.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    out = torch.matmul(p[..., :T].reshape(H, B * tq * G, T), st.shared_v[l].float()).reshape(H, B, tq, G, D).permute(1, 2, 0, 3, 4)
    rest = torch.matmul(p[..., T:].permute(1, 0, 2, 3, 4).reshape(B, H, tq * G, N + tq), v).reshape(B, H, tq, G, D)
    out = out + rest.permute(0, 2, 1, 3, 4)
    moved = []
    for x in (k, v):
        x = x[:, :, tq:]
        W = c["window"]
        if 0 <= W < N:
            lo = max(0, N - W - tq)
            x = torch.cat([x[:, :, :lo], _codes(x[:, :, lo:N - W]), x[:, :, N - W:]], 2)
        moved.append(x)
    st.rows[l] = moved
    return out.reshape(B, tq, Hq, D).half()


# ---- logits ----

def _run_constrain(st):
    c = st.case
    if own:
        st.kv.constrain(st.logits, st.out, tokens=st.tokens, lengths=st.lengths, prompt_lengths=st.prompt_lengths,
                        repetition=st.repetition, presence=st.presence, frequency=st.frequency, bias_offsets=st.bias_offsets,
                        bias_tokens=st.bias_tokens, bias_values=st.bias_values, allowed=st.allowed)
        return st.out
    B, V = c["batch"], c["vocab"]
    at = torch.arange(st.tokens.shape[1], device="cuda")
    there, said = (at < st.lengths[:, None]), (at >= st.prompt_lengths[:, None])
    ids = st.tokens.long()
    count = torch.zeros(B, V, dtype=torch.int32, device="cuda").scatter_add_(1, ids, (there & said).int())
    seen = torch.zeros(B, V, dtype=torch.int32, device="cuda").scatter_add_(1, ids, there.int()) > 0
    x = st.logits.float()
    r = st.repetition[:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - st.frequency[:, None] * count - st.presence[:, None] * (count > 0)
    row = torch.arange(B, device="cuda").repeat_interleave(c["bias"])
    x[row, st.bias_tokens.long()] += st.bias_values
    if st.allowed is not None:
        bits = (st.allowed[..., None] >> torch.arange(32, device="cuda")) & 1
        x = x.masked_fill(bits.reshape(B, -1)[:, :V] == 0, -math.inf)
    return x


# ---- the same in 64 bits ----

def exact(c, seed):
    return {"prepare": _exact_prepare, "shared": _exact_shared, "constrain": _exact_constrain}[c["op"]](c, seed)


def _exact_prepare(c, seed):
    """Pairs as complex numbers, turned by e^(i angle)."""
    st = _prepare_inputs(c, seed)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st.pos.double()[..., None] * st.freq.double())[:, :, None]
    R, got = c["rotated"], {}
    for name, x, w in (("q", st.q, st.wq), ("k", st.k, st.wk)):
        x = x.double()
        if w is not None:
            x = x / ((x ** 2).sum(-1, keepdim=True) / c["dim"] + EPS).sqrt() * w.double()
        first, second = (x[..., 0:R:2], x[..., 1:R:2]) if c["paired"] else x[..., :R].chunk(2, -1)
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        y = x.clone()
        if c["paired"]:
            y[..., 0:R:2], y[..., 1:R:2] = z.real, z.imag
        else:
            y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
        got[name] = y
    got["v"] = st.v.double()
    if c["prompt"]:
        got["k"], got["v"] = (got[n].permute(0, 2, 1, 3).contiguous() for n in ("k", "v"))
    return got


def _exact_shared(c, seed):
    """Sequence by sequence: the rows it sees laid end to end."""
    st = _shared_inputs(c, seed)
    L, B, tq, Hq, H, D, N = (c[k] for k in ("layers", "batch", "tokens", "heads", "kv_heads", "dim", "cache"))
    G, W, seen = Hq // H, c["window"], _seen(c)
    out = torch.empty(L, B, tq, Hq, D, dtype=torch.float64, device="cuda")

    def rows(shared, cache, new, l, b):
        x = cache[l, b].double()
        if W >= 0 and N > W:
            x = x.clone()
            o = x[:, :N - W]
            s = (o.abs().amax(-1, keepdim=True).float() / 127.0).half().double()
            x[:, :N - W] = torch.where(s > 0, (o / s.clamp(min=1e-300)).round().clamp(-127, 127) * s, 0.0)
        return torch.cat([shared[l, :, :seen[b]].double(), x, new[l, b].permute(1, 0, 2).double()], 1)

    for l in range(L):
        for b in range(B):
            k, v = rows(st.shared_k, st.cache_k, st.k, l, b), rows(st.shared_v, st.cache_v, st.v, l, b)
            n = k.shape[1]
            for h in range(H):
                q = st.q[l, b, :, h * G:(h + 1) * G].double().reshape(tq * G, D)
                s = (q @ k[h].T.contiguous()) * float(torch.tensor(1.0 / math.sqrt(D)))
                last = (n - tq + torch.arange(tq, device="cuda")).repeat_interleave(G)
                s = s.masked_fill(torch.arange(n, device="cuda") > last[:, None], -math.inf)
                out[l, b, :, h * G:(h + 1) * G] = (torch.softmax(s, -1) @ v[h]).reshape(tq, G, D)
    return out


def _exact_constrain(c, seed):
    """Row by row, with a bincount."""
    st = _constrain_inputs(c, seed)
    V, m = c["vocab"], c["bias"]
    rows = []
    for b in range(c["batch"]):
        n, first = int(st.lengths[b]), int(st.prompt_lengths[b])
        x = st.logits[b].double()
        everywhere = torch.bincount(st.tokens[b, :n].long(), minlength=V)
        said = torch.bincount(st.tokens[b, first:n].long(), minlength=V)
        r, f, p = (float(t[b]) for t in (st.repetition, st.frequency, st.presence))
        again = everywhere > 0
        x[again & (x > 0)] /= r
        x[again & (x < 0)] *= r
        x -= f * said.double()
        x[said > 0] -= p
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        bias[st.bias_tokens[b * m:(b + 1) * m].long()] = st.bias_values[b * m:(b + 1) * m].double()
        x += bias
        if st.bits is not None:
            x[~st.bits[b, :V]] = -math.inf
        rows.append(x)
    return torch.stack(rows)
