"""Timed cases of the cache held in 8 bits and of attention with a sliding window: rows coded as they are written and read back,
attention of new tokens and of chunks of a prompt over the coded cache, and over the plain one with a window of the newest tokens
and a few first ones (sinks).

Each operator is here in two forms: its plain one (elementary torch operations in 32 bits, 64 where 32 lose what matters) and,
with ``own`` set, the call a program makes of this package.  Keys have the statistics of the package's own workloads:
Gaussian rows with four strong channels per KV head; every query leans towards one of the keys it sees.

The coded cache: 64 neighbouring tokens of a KV head are a block.  A block that is full is held as 8-bit codes with one scale for its keys
and one for its values; the rows behind the last full block are held as they are.
  int8   scale = amax / 127, rounded to 32 bits and then to 16 significant ones; code = the integer nearest to x / scale, ties to even
  e4m3   scale = the smallest power of two with amax <= 448 scale; code = x / scale rounded to e4m3
A row reads as code * scale.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH_DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 64                         # tokens of a block of the coded cache
TINY = 2.0 ** -100                 # a block whose largest number is below is held as zeros


def _case(name, op, *, tokens, seqs=1, q_heads=32, kv_heads=8, dim=128, dtype="bf16", **more):
    case = dict(op=op, tokens=tokens, seqs=seqs, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, ragged=False)
    case.update(dict(format="int8", step=0, heads_first=False) if op == "store" else
                dict(format="int8" if op == "coded" else "", queries=1, window=0, sinks=0))
    case.update(more)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # 64 steps of generation of 16 sequences, a token each, then what they hold
        _case("store_steps64_batch16_int8", "store", tokens=64, seqs=16, step=1),
        # a prompt of odd length into the cache, and all of it read back (a cache that changes hands)
        _case("store_prompt_8k_e4m3_f16", "store", tokens=8191, dtype="f16", format="e4m3"),
        # four long documents imported head by head from another cache, and read back
        _case("store_batch4_48k_int8", "store", tokens=48001, seqs=4, heads_first=True, ragged=True),
        # one new token of a short chat, all latency
        _case("coded_500_int8", "coded", tokens=500),
        # a batch of requests of different length
        _case("coded_batch16_32k_e4m3_f16", "coded", tokens=32768, seqs=16, q_heads=64, ragged=True, dtype="f16", format="e4m3"),
        # one new token at a million tokens: the most that is read
        _case("coded_1m_int8_f16", "coded", tokens=1048577, dtype="f16"),
        # the last 2048 tokens of a long prompt that is filled in chunk by chunk
        _case("coded_chunk2k_at_24k_int8", "coded", tokens=24000, queries=2048),
        # one new token of a long chat in a layer with a window
        _case("sinks_32k_w1k", "sinks", tokens=32768, window=1024, sinks=4),
        # a batch far into its contexts, a wide window
        _case("sinks_batch16_64k_w4k_f16", "sinks", tokens=65536, seqs=16, q_heads=64, ragged=True, window=4096, sinks=128, dtype="f16"),
        # eight drafted tokens of four sequences, verified against all that is cached
        _case("prompt_draft8_batch4_20k", "prompt", tokens=20011, seqs=4, queries=8, ragged=True),
        # a whole prompt, every token sees all before it
        _case("prompt_8k", "prompt", tokens=8192, queries=8192),
        # a long prompt of odd length in a layer with a window
        _case("prompt_16k_w2k_f16", "prompt", tokens=16001, queries=16001, q_heads=16, kv_heads=4, window=2048, sinks=16, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 8), (32, 8), (64, 8), (16, 2), (28, 4), (16, 16), (16, 1), (8, 2)]       # (query, KV) heads of models in use


def draw(rng):
    op = rng.choice(["store", "coded", "coded", "coded_chunk", "sinks", "prompt", "prompt"])
    hq, hkv = rng.choice(HEADS)
    dtype, dim = rng.choice(["f16", "bf16", "f16", "bf16", "f32"]), rng.choice([32, 64, 128, 128, 128, 256])
    shape = dict(q_heads=hq, kv_heads=hkv, dim=dim, dtype=dtype)
    fmt = rng.choice(["int8", "e4m3"])
    row = hkv * dim * BYTES[dtype]
    seqs = rng.choice([1, 1, 1, 2, 5, _log_int(rng, 2, 64)])
    ragged = seqs > 1 and rng.random() < 0.7
    if op == "store":
        if rng.random() < 0.4:
            return _case("", op, tokens=rng.randint(20, 150), seqs=min(seqs, 16), step=1, format=fmt, **shape)
        seqs = min(seqs, 8)
        tokens = min(_log_int(rng, 32, 131072), max(32, (1 << 28) // (row * seqs)))
        return _case("", op, tokens=tokens, seqs=seqs, ragged=ragged, heads_first=rng.random() < 0.4, format=fmt, **shape)
    if op in ("coded", "sinks"):
        tokens = min(_log_int(rng, 16, 524288), max(16, (1 << 30) // (row * seqs)))
        win = op == "sinks" or rng.random() < 0.25
        window = min(tokens, _log_int(rng, 16, 16384)) if win else 0
        return _case("", op, tokens=tokens, seqs=seqs, ragged=ragged, window=window, sinks=rng.choice([0, 1, 4, 100]) if win else 0,
                     **({"format": fmt} if op == "coded" else {}), **shape)
    queries = rng.choice([_log_int(rng, 2, 64), _log_int(rng, 16, 8192)])
    # keys and queries of a size that the plain form's scores fit: 2^30 numbers, a quarter of the largest listed case's
    most = max(queries, (1 << 30) // (hq * seqs * queries))
    while seqs * hq * queries * queries > 1 << 30:
        seqs, queries = max(1, seqs // 2), queries if seqs > 1 else queries * 2 // 3
        most = max(queries, (1 << 30) // (hq * seqs * queries))
    tokens = min(queries + rng.choice([0, 0, _log_int(rng, 1, 65536)]), most, max(queries, (1 << 29) // (row * seqs)))
    window = rng.choice([0, 0, min(tokens, _log_int(rng, 16, 8192))])
    return _case("", "coded" if op == "coded_chunk" else op, tokens=tokens, seqs=seqs, queries=queries, ragged=seqs > 1 and ragged and tokens > queries,
                 window=window, sinks=rng.choice([0, 1, 4, 100]) if window else 0, **({"format": fmt} if op == "coded_chunk" else {}), **shape)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def lengths(case):
    """Tokens of every sequence: all alike, or spread between a twentieth and the whole of `tokens` in a fixed irregular order."""
    n = case["tokens"]
    if not case["ragged"]:
        return [n] * case["seqs"]
    least = max(1, case.get("queries", 1))
    return [max(least, n - (b * 7919 % 1009) * (n - n // 20) // 1009) for b in range(case["seqs"])]


def _window(case):
    return case["window"] or case["tokens"]                            # 0: all tokens


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(((seed & 0x7FFFFFFF) << 24) + stream)
    return g


def _keys_values(case, seed, seq, n):
    """K, V [Hkv, n, d] of one sequence, rounded to the rows' type."""
    g = _generator(seed, 0x1000 + seq)
    Hkv, d, dt = case["kv_heads"], case["dim"], TORCH_DTYPE[case["dtype"]]
    V = torch.randn((Hkv, n, d), generator=g, device="cuda").to(dt)
    K = torch.randn((Hkv, n, d), generator=g, device="cuda")
    strong = torch.rand((Hkv, d), generator=g, device="cuda").argsort(1)[:, :4]
    K *= torch.ones((Hkv, d), device="cuda").scatter_(1, strong, 3.0)[:, None]
    return K.to(dt), V


def _queries(case, seed, seq, K):
    """[M, Hq, d] for the last M of the n tokens K [Hkv, n, d]: Gaussian, leaning towards one of the keys that each sees."""
    g = _generator(seed, 0x4000 + seq)
    M, Hq, Hkv, d, n = case["queries"], case["q_heads"], case["kv_heads"], case["dim"], K.shape[1]
    q = torch.randn((M, Hq, d), generator=g, device="cuda")
    pos = torch.arange(n - M, n, device="cuda")[:, None]
    back = torch.rand((M, Hq), generator=g, device="cuda") * torch.clamp(pos + 1, max=_window(case))
    at = (pos - back.long()).clamp(min=0)
    head = (torch.arange(Hq, device="cuda") // (Hq // Hkv)).expand(M, Hq)
    q += 6.0 * math.sqrt(d) / (d + 32.0) * K[head, at].float()
    return q.to(TORCH_DTYPE[case["dtype"]])


def _rows_in(case, seed, seq, n):
    """The same rows as a program has them before they are cached, [n, Hkv, d]: views of one fused projection, or of another cache's heads."""
    K, V = _keys_values(case, seed, seq, n)
    if case["heads_first"]:
        return K.transpose(0, 1), V.transpose(0, 1)
    fused = torch.cat([K, V], 0).transpose(0, 1).contiguous()
    return fused[:, :case["kv_heads"]], fused[:, case["kv_heads"]:]


def prepare(case, seed):
    op, B, Hq, Hkv, d, cap = (case[x] for x in ("op", "seqs", "q_heads", "kv_heads", "dim", "tokens"))
    dt = TORCH_DTYPE[case["dtype"]]
    state = dict(case=case, lens=lengths(case))
    if op == "store":
        rows = [_rows_in(case, seed, b, n) for b, n in enumerate(state["lens"])]
        state["src"] = [tuple(torch.stack([r[i] for r in rows]) for i in range(2))] if case["step"] else [(k[None], v[None]) for k, v in rows]
    else:
        q = []
        for b, n in enumerate(state["lens"]):
            q.append(_queries(case, seed, b, _keys_values(case, seed, b, n)[0]))
        state["q"] = torch.stack(q) if case["queries"] > 1 else torch.stack(q)[:, 0]
    if own:
        from paper_2502_06766_amd import topk_attn as ta
        types = {"f32": ta.F32, "f16": ta.F16, "bf16": ta.BF16}
        if op in ("store", "coded"):
            cache = ta.TopkAttnCodedCache(1, B, Hq, Hkv, d, cap, types[case["dtype"]],
                                          format={"int8": ta.CODED_INT8, "e4m3": ta.CODED_E4M3}[case["format"]])
        else:
            cache = ta.TopkAttnCache(1, B, Hq, Hkv, d, cap, 64, types[case["dtype"]])
        state["cache"] = cache
        for b, n in enumerate(state["lens"] if op != "store" else []):
            K, V = _keys_values(case, seed, b, n)
            if op == "coded":
                cache.append(0, K.transpose(0, 1)[None], V.transpose(0, 1)[None], seq=b)
            else:
                cache.append(0, b, K, V, head_major=True)
        return state
    if op in ("store", "coded"):
        state["codes"], state["scales"], state["open"] = _coded_cache(case)
        for b, n in enumerate(state["lens"] if op == "coded" else []):
            K, V = _keys_values(case, seed, b, n)
            _append(state, slice(b, b + 1), 0, K[None], V[None])
    else:
        state["K"], state["V"] = (torch.zeros((B, Hkv, cap, d), dtype=dt, device="cuda") for _ in range(2))
        for b, n in enumerate(state["lens"]):
            state["K"][b, :, :n], state["V"][b, :, :n] = _keys_values(case, seed, b, n)
    state["n"] = torch.tensor(state["lens"], device="cuda")
    return state


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    case, cache = state["case"], state["cache"]
    if case["op"] == "store":
        cache.reset(0)
        if case["step"]:
            K, V = state["src"][0]
            for t in range(0, case["tokens"], case["step"]):
                cache.append(0, K[:, t:t + case["step"]], V[:, t:t + case["step"]])
            return cache.read(0, 0, case["tokens"])
        for b, (K, V) in enumerate(state["src"]):
            cache.append(0, K, V, seq=b)
        return [cache.read(0, 0, n, seq=b) for b, n in enumerate(state["lens"])]
    window = _window(case)
    if case["queries"] > 1:
        return cache.prompt(0, state["q"], window=window, sinks=case["sinks"])
    if case["op"] == "coded":
        return cache.decode(0, state["q"], window=window, sinks=case["sinks"])
    return cache.decode_sinks(0, state["q"], window=window, sinks=case["sinks"])


def _run_plain(state):
    case = state["case"]
    B, Hkv, d, cap, dt = case["seqs"], case["kv_heads"], case["dim"], case["tokens"], TORCH_DTYPE[case["dtype"]]
    if case["op"] == "store":
        if case["step"]:
            K, V = (x.transpose(1, 2) for x in state["src"][0])
            for t in range(0, cap, case["step"]):
                _append(state, slice(0, B), t, K[:, :, t:t + case["step"]], V[:, :, t:t + case["step"]])
            return tuple(x.transpose(1, 2).to(dt) for x in _decoded(state, slice(0, B), cap))
        for b, (K, V) in enumerate(state["src"]):
            _append(state, slice(b, b + 1), 0, K.transpose(1, 2), V.transpose(1, 2))
        return [tuple(x.transpose(1, 2).to(dt) for x in _decoded(state, slice(b, b + 1), n)) for b, n in enumerate(state["lens"])]
    if case["op"] == "coded":
        K, V = (x[:, :, :cap] for x in _decoded(state, slice(0, B), cap, state["n"]))
    else:
        K, V = state["K"].float(), state["V"].float()
    M = case["queries"]
    q = state["q"].float().view(B, M, Hkv, -1, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)          # rows: head of the group, query
    token = torch.arange(cap, device="cuda")
    pos = (state["n"][:, None] - M + torch.arange(M, device="cuda"))[:, :, None]                           # [B, M, 1]
    hidden = (token > pos) | ((token <= pos - _window(case)) & (token >= case["sinks"]))
    s = torch.matmul(q, K.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(B, -1, M, cap)
    s.masked_fill_(hidden[:, None], -math.inf)
    top = s.amax(3, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(3, keepdim=True)
    out = torch.matmul(s.view(B, Hkv, -1, cap), V).view(B, -1, M, d) / total
    out, lse = out.transpose(1, 2), (top + torch.log(total))[..., 0].transpose(1, 2)
    return (out[:, 0], lse[:, 0]) if M == 1 else (out.to(dt), lse)


# ---- the coded cache in its plain form --------------------------------------------------------------------------------
def _coded_cache(case):
    """Codes, scales and open rows, each a pair for keys and values."""
    B, Hkv, d = case["seqs"], case["kv_heads"], case["dim"]
    P = (case["tokens"] + BLOCK - 1) // BLOCK
    kind = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    codes = [torch.zeros((B, Hkv, P, BLOCK, d), dtype=kind, device="cuda") for _ in range(2)]
    scales = [torch.zeros((B, Hkv, P), device="cuda") for _ in range(2)]
    rows = [torch.zeros((B, Hkv, BLOCK, d), dtype=TORCH_DTYPE[case["dtype"]], device="cuda") for _ in range(2)]
    return codes, scales, rows


def _code(fmt, x):
    """x [..., blocks, 64, d] -> codes, scales [..., blocks]."""
    amax = x.abs().amax((-2, -1)).float()
    if fmt == "int8":
        bits = (amax / 127.0).view(torch.int32)
        scale = ((bits + 0x7F + ((bits >> 8) & 1)) & -256).view(torch.float32)
    else:
        part, power = torch.frexp(amax)
        scale = ((power - 9 + (part > 0.875).int()).clamp(min=-126) + 127 << 23).view(torch.float32)       # that power of two
    scale = torch.where(amax < TINY, 0.0, scale)
    by = torch.where(scale > 0, scale, 1.0)[..., None, None]
    live = (scale > 0)[..., None, None]
    if fmt == "int8":
        return torch.where(live, torch.round(x.double() / by.double()), 0.0).to(torch.int8), scale
    return torch.where(live, x.float() / by, 0.0).to(torch.float8_e4m3fn), scale


def _append(state, seqs, n0, K, V):
    """Rows [S, Hkv, n, d] behind the n0 that the sequences hold."""
    held, p0 = n0 % BLOCK, n0 // BLOCK
    for i, x in enumerate((K, V)):
        rows = state["open"][i][seqs]
        x = torch.cat([rows[:, :, :held], x], 2) if held else x
        full = x.shape[2] // BLOCK
        if full:
            blocks = x[:, :, :full * BLOCK].reshape(*x.shape[:2], full, BLOCK, -1)
            codes, scales = _code(state["case"]["format"], blocks)
            state["codes"][i][seqs, :, p0:p0 + full], state["scales"][i][seqs, :, p0:p0 + full] = codes, scales
        rows[:, :, :x.shape[2] - full * BLOCK] = x[:, :, full * BLOCK:]


def _decoded(state, seqs, n, each=None):
    """Keys and values [S, Hkv, n, d] in 32 bits (`each`: of sequences with so many tokens; zero behind them)."""
    got = []
    for i in range(2):
        x = state["codes"][i][seqs].float() * state["scales"][i][seqs][..., None, None]
        S, Hkv, P, _, d = x.shape
        x, rows = x.view(S, Hkv, P * BLOCK, d), state["open"][i][seqs].float()
        if each is None:
            x[:, :, n // BLOCK * BLOCK:n] = rows[:, :, :n % BLOCK]
        else:
            at = (each // BLOCK * BLOCK)[:, None] + torch.arange(BLOCK, device="cuda")               # [S, 64] places of the open rows
            there = (at < each[:, None])[:, None, :, None]
            at = at.clamp(max=P * BLOCK - 1)[:, None, :, None].expand(S, Hkv, BLOCK, d)
            x.scatter_(2, at, torch.where(there, rows, x.gather(2, at)))
        got.append(x[:, :, :n])
    return got


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    B, Hq, Hkv, d, e, M = case["seqs"], case["q_heads"], case["kv_heads"], case["dim"], BYTES[case["dtype"]], case.get("queries", 1)
    lens = lengths(case)
    if case["op"] == "store":
        full = sum(n // BLOCK * BLOCK for n in lens)
        # rows read; codes of the full blocks written and read, open rows too; rows written
        moved = 2 * Hkv * d * (2 * sum(lens) * e + 2 * full + 2 * (sum(lens) - full) * e) + 16 * Hkv * (full // BLOCK) * 2
        return {"bytes": moved, "flops": 4 * 2 * full * Hkv * d}
    window, sinks = _window(case), case["sinks"]
    read = pairs = 0
    for n in lens:
        first = max(0, n - M - window + 1)                             # the oldest token of a window
        read += n - first + min(sinks, first)
        # sum over the queries' positions p of min(p + 1, window + the sinks before the window)
        short = max(0, min(n, window) - (n - M))                       # queries that see all before them
        pairs += short * (n - M + 1) + short * (short - 1) // 2 + sum(window + min(sinks, p + 1 - window) for p in range(n - M + short, n))
    size = 1 if case["op"] == "coded" else e
    ends = B * M * Hq * (d * e + d * (4 if M == 1 else e) + 4)
    return {"bytes": 2 * read * Hkv * d * size + ends, "flops": 4 * pairs * Hq * d}


# ---- reference in 64 bits ---------------------------------------------------------------------------------------------
def _power64(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _held64(fmt, x):
    """x [H, n, d] as the coded cache holds it, in 64 bits."""
    y, n = x.double(), x.shape[1]
    full = n // BLOCK * BLOCK
    for h in range(x.shape[0] if full else 0):
        z = y[h, :full].view(-1, BLOCK * x.shape[2])
        amax = z.abs().max(1, keepdim=True).values
        if fmt == "int8":
            m, p = torch.frexp((amax / 127.0).float().double())
            m = m * 65536.0                                            # 16 significant bits, ties to even
            low = torch.floor(m)
            up = (m - low > 0.5) | ((m - low == 0.5) & (low % 2 == 1))
            scale = (low + up) / 65536.0 * _power64(p)
            t = z / torch.where(amax < TINY, 1.0, scale)
            low = torch.floor(t)
            up = (t - low > 0.5) | ((t - low == 0.5) & (low % 2 == 1))
            held = (low + up) * scale
        else:
            p = torch.ceil(torch.log2(amax / 448.0)).clamp(min=-140)
            p = p + (amax > 448.0 * _power64(p)).double() - (amax <= 448.0 * _power64(p - 1)).double()
            scale = _power64(p)
            t = z / scale
            step = _power64(torch.frexp(t)[1].clamp(min=-5) - 4)                   # spacing of e4m3: 3 bits behind the first, 2^-9 at the least
            low = torch.floor(t / step)
            rest = t / step - low
            held = (low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 == 1)))) * step * scale
        y[h, :full] = torch.where(amax < TINY, 0.0, held).view(full, -1)
    return y


def exact(case, seed):
    Hq, Hkv, d, M = case["q_heads"], case["kv_heads"], case["dim"], case.get("queries", 1)
    G, lens = Hq // Hkv, lengths(case)
    if case["op"] == "store":
        got = [tuple(_held64(case["format"], x).transpose(0, 1) for x in _keys_values(case, seed, b, n)) for b, n in enumerate(lens)]
        if case["step"]:
            return tuple(torch.stack([r[i] for r in got]) for i in range(2))
        return [(k[None], v[None]) for k, v in got]
    outs, lses = [], []
    for b, n in enumerate(lens):
        K, V = _keys_values(case, seed, b, n)
        q = _queries(case, seed, b, K).double()                        # [M, Hq, d]
        out = torch.empty((M, Hq, d), dtype=torch.float64, device="cuda")
        lse = torch.empty((M, Hq), dtype=torch.float64, device="cuda")
        back = torch.arange(n - M, n, device="cuda")[:, None] - torch.arange(n, device="cuda")        # tokens between query and key
        seen = (back >= 0) & ((back < _window(case)) | (torch.arange(n, device="cuda") < case["sinks"]))
        for h in range(Hq):
            if h % G == 0:
                k, v = (x[h // G:h // G + 1] for x in (K, V))
                k, v = (_held64(case["format"], x)[0] if case["op"] == "coded" else x[0].double() for x in (k, v))
            s = torch.where(seen, (q[:, h] @ k.t()) / math.sqrt(d), -math.inf)
            lse[:, h] = torch.logsumexp(s, 1)
            out[:, h] = torch.exp(s - lse[:, h, None]) @ v
        outs.append(out)
        lses.append(lse)
    out, lse = torch.stack(outs), torch.stack(lses)
    return (out[:, 0], lse[:, 0]) if M == 1 else (out, lse)
