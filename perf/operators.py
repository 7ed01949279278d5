"""The operators around a quantised K/V cache and several new tokens at a time, as cases to be timed.

quant   K/V rows of a step or a prompt are written into the microscaled cache and read back from it
sparse  one decode step's attention over the retrieved rows of a quantised cache
tiered  the same with Sink + Local + Update Buffer rows from the float16 window cache, the records in pinned host memory
tree    attention of a tree of drafted tokens over the cached rows (float16 or quantised) and the drafts
sink    attention of new tokens over a sliding window and the first tokens, which stay visible

A block of 32 dimensions of a row has one scale 2^s, s the smallest integer >= s_min with amax <= M 2^s, and a code a
value: the nearest of 8-bit e4m3 (M = 448, s_min = -15) or 4-bit e2m1 (M = 6, s_min = -23), ties to the even code, no
value past 65504.  A record holds a row's K codes, V codes, 4 + 4 scale bytes s + 127, and zeros up to 16 bytes.

Keys follow the workloads' law: a mean offset per channel, unit scale except 4 outlier channels at 8; values N(0, 1);
a query is a planted key plus noise or a draw from the key law.
"""

import hashlib
import math

import numpy as np
import torch

own = False

D, BLOCK = 128, 32
SINK, LOCAL, UPDATE = 128, 512, 256  # region sizes of the decode loop
SCALE = D ** -0.5


def _case(op, name, batch, hkv, g, n, **more):
    """n: rows of the cache; t: new rows (quant), drafted tokens (tree), new tokens (sink)."""
    c = dict(op=op, batch=batch, hkv=hkv, g=g, n=n, kbits=8, vbits=8, t=1, k=0, query="needle", ragged=False)
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One decode step's rows of 4 sequences, each at a length of its own: latency.
        _case("quant", "quant_step", 4, 8, 4, 33000, t=1, ragged=True),
        # Prefill of a few prompts of no round length, 8-bit keys and 4-bit values.
        _case("quant", "quant_ragged", 3, 8, 4, 10007, t=10007, vbits=4),
        # Prefill of one layer at 128K tokens.
        _case("quant", "quant_128k", 1, 8, 4, 131072, t=131072),
        # The retrieved rows of one sequence at 32K tokens: latency.
        _case("sparse", "sparse_32k", 1, 8, 4, 32768, k=256),
        # Throughput: 8 sequences at 128K tokens, 8-bit keys and 4-bit values.
        _case("sparse", "sparse_8x128k", 8, 8, 4, 131072, k=512, vbits=4, query="law"),
        # A step of the offload setting: 4-bit records in pinned host memory, a partly filled update buffer.
        _case("tiered", "tiered_host_128k", 1, 8, 4, 131072, k=512, kbits=4, vbits=4, buffered=200),
        # The smallest verification: one KV head, 8 drafted tokens over 4096 rows.
        _case("tree", "tree_tiny", 1, 1, 8, 4096, t=8, kbits=16, vbits=16),
        # A long generation with drafts: 4 sequences of any length over an 8-bit cache.
        _case("tree", "tree_ragged", 4, 8, 4, 45679, t=31, ragged=True, query="law"),
        # Throughput: 16 drafts of 8 sequences at 128K tokens.
        _case("tree", "tree_8x128k", 8, 8, 4, 131072, t=16, kbits=16, vbits=16),
        # One token of a wide batch of short contexts with a head count that is no multiple of 4.
        _case("sink", "sink_step", 16, 4, 7, 7001, t=1, sink=4, window=4096, ragged=True, query="law"),
        # A few prompts of different lengths, padded to the longest.
        _case("sink", "sink_ragged", 3, 8, 4, 2501, t=2501, sink=128, window=512, ragged=True, query="law"),
        # The last chunk of a long prompt.
        _case("sink", "sink_chunk", 1, 8, 4, 16384, t=8192, sink=128, window=4096, query="law"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quant", "quant", "sparse", "sparse", "tiered", "tree", "tree", "tree", "sink", "sink", "sink"])
    hkv, g = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    batch = _log_int(rng, 1, 16)
    rows = batch * hkv
    bits = dict(zip(("kbits", "vbits"), rng.choice([(8, 8), (8, 8), (8, 4), (4, 4), (4, 8)])))
    query = rng.choice(["needle", "law"])
    if op == "quant":
        t = _log_int(rng, 1, max(1, min(131072, (1 << 20) // rows)))
        return _case(op, None, batch, hkv, g, t + rng.randrange(100), t=t, ragged=rng.random() < 0.5, **bits)
    if op in ("sparse", "tiered"):
        n = _log_int(rng, 512, max(512, min(131072, (1 << 22) // rows)))
        k = max(1, min(n, rng.choice([32, 64, 100, 256, 512, 1024]), (16384 if op == "tiered" else 1 << 17) // (rows * g)))
        more = dict(buffered=rng.randrange(UPDATE)) if op == "tiered" else {}
        return _case(op, None, batch, hkv, g, n, k=k, query=query, ragged=rng.random() < 0.3, **more, **bits)
    if op == "tree":
        if rng.random() < 0.5:
            bits = dict(kbits=16, vbits=16)
        t = rng.choice([1, 2, 5, 8, 16, 31, 48, 64])
        n = _log_int(rng, 64, max(64, min(131072, (1 << 23) // rows, (1 << 29) // (rows * g * t))))
        return _case(op, None, batch, hkv, g, n, t=t, query=query, ragged=rng.random() < 0.5, **bits)
    t = rng.choice([1, 1, 4, 16]) if rng.random() < 0.4 else _log_int(rng, 32, max(32, min(8192, (1 << 15) // (rows * g) * 8)))
    n = t + (_log_int(rng, 1, max(1, min(32768, (1 << 32) // (rows * g * t) - t))) if rng.random() < 0.7 else 0)
    window = _log_int(rng, 16, max(16, min(16384, (1 << 30) // (rows * g * t))))
    return _case(op, None, batch, hkv, g, n, t=t, sink=rng.choice([0, 4, 64, 128]), window=window, query=query,
                 ragged=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs


def _seed(case, seed):
    text = ",".join(f"{k}={case[k]}" for k in sorted(case) if k != "name") + f",{seed}"
    return int.from_bytes(hashlib.sha256(text.encode()).digest()[:7], "little")


def _record(case):
    """(bytes of K codes, of V codes, of a record)"""
    kb, vb = D * case["kbits"] // 8, D * case["vbits"] // 8
    return kb, vb, -(-(kb + vb + 8) // 16) * 16


def _ancestors(rng, batch, t):
    """Masks of random trees: a token sees itself and the path to its root."""
    bits = np.zeros((batch, t, t), dtype=bool)
    for b in range(batch):
        for i in range(t):
            parent = int(rng.integers(-1, i)) if i else -1
            if parent >= 0:
                bits[b, i] = bits[b, parent]
            bits[b, i, i] = True
    return (bits.astype(np.uint64) << np.arange(t, dtype=np.uint64)).sum(2, dtype=np.uint64).view(np.int64)


def prepare(case, seed):
    s = _seed(case, seed)
    gen, rng = torch.Generator(device="cuda").manual_seed(s), np.random.default_rng(s)
    b, h, g, n, t, op = (case[k] for k in ("batch", "hkv", "g", "n", "t", "op"))

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    mu = 0.5 * randn(b, h, 1, D)
    scale = torch.ones(b, h, 1, D, device="cuda")
    scale.scatter_(3, torch.rand(b, h, 1, D, generator=gen, device="cuda").argsort(dim=3)[..., :4], 8.0)

    def kv(rows):
        return randn(b, h, rows, D).mul_(scale).add_(mu).half(), randn(b, h, rows, D).half()

    st = dict(case=case)
    K, V = kv(t if op == "quant" else n)
    if op == "quant":
        st["K"], st["V"] = K, V
        st["rec"] = torch.zeros(b, h, n, _record(case)[2], dtype=torch.uint8, device="cuda")
        # Each sequence's first new row, where the sequences differ in length, and where they do not.
        st["rows"] = torch.from_numpy(rng.integers(0, n - t + 1, b).astype(np.int32)).cuda() if case["ragged"] else None
        st["outs"] = tuple(torch.empty(b, h, t, D, dtype=torch.float16, device="cuda") for _ in range(2))
        return st
    tokens = t if op in ("tree", "sink") else 1
    if case["query"] == "needle":
        at = torch.randint(0, n, (b, h, g * tokens, 1), generator=gen, device="cuda").expand(b, h, g * tokens, D)
        q = (torch.gather(K, 2, at).float() + 0.1 * randn(b, h, g * tokens, D)).half()
    else:
        q = (mu + scale * randn(b, h, g * tokens, D)).half()
    st["q"] = q.reshape((b, h * g, tokens, D) if op in ("tree", "sink") else (b, h * g, D))
    st["out"] = torch.zeros(st["q"].shape, dtype=torch.float16 if op == "sink" else torch.float32, device="cuda")
    if op != "sink" and case["kbits"] < 16:
        st["rec"] = _pack(case, K, V)
    else:
        st["K"], st["V"] = K, V
    if op in ("sparse", "tiered"):
        k = case["k"]
        idx = torch.rand(b, h * g, n, generator=gen, device="cuda").topk(k).indices.sort().values.int()
        if case["ragged"]:  # some heads found fewer rows
            idx[:, ::2, k - k // 3:] = -1
        st["idx"] = idx
    if op == "tiered":
        begin = SINK + n
        end = begin + LOCAL + case["buffered"]
        st["win"] = (SINK, SINK, begin, end)
        st["K_win"], st["V_win"] = kv(SINK + LOCAL + UPDATE)
        rec = torch.zeros(b, h, begin, st["rec"].shape[3], dtype=torch.uint8, device="cuda")
        rec[:, :, SINK:] = st["rec"]
        st["rec"] = torch.empty(rec.shape, dtype=torch.uint8, pin_memory=True).copy_(rec)
    if op == "tree":
        st["K_tree"], st["V_tree"] = kv(t)
        st["mask"] = torch.from_numpy(_ancestors(rng, b, t)).cuda()
        st["lens"] = torch.from_numpy(rng.integers(n // 2, n + 1, b).astype(np.int32)).cuda() if case["ragged"] else None
    if op == "sink":
        # Sequences of different lengths: a prompt ends earlier, a later chunk or a single token begins earlier.
        prompt = case["ragged"] and n == t
        st["counts"] = torch.from_numpy(rng.integers((t + 1) // 2, t + 1, b).astype(np.int32)).cuda() if prompt else None
        st["starts"] = torch.from_numpy(rng.integers((n - t) // 2, n - t + 1, b).astype(np.int32)).cuda() if (
            case["ragged"] and not prompt) else None
    return st


# ---------------------------------------------------------------- the plain forms


def _pow2(s):
    return ((s + 127) << 23).view(torch.float32)


def _quantized(x, bits):
    """(code values y, exponents s) of x [..., D]: the row stands for y 2^s, block by block."""
    top, mant, s_min, lowest, s_max, most = (1.75, 3, -15, -6, 8, 240.0) if bits == 8 else (1.5, 1, -23, 0, 14, 3.0)
    x = x.float().reshape(*x.shape[:-1], D // BLOCK, BLOCK)
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    s = torch.where(m > 0, e - 1 - (8 if bits == 8 else 2) + (2 * m > top).int(), s_min).clamp(min=s_min).int()
    y = x * _pow2(-s)
    step = _pow2((torch.frexp(y)[1] - 1).clamp(min=lowest).int() - mant)
    y = torch.round(y / step) * step
    limit = torch.where(s == s_max, most, 448.0)
    return torch.minimum(torch.maximum(y, -limit), limit), s


def _codes(y, bits):
    """The codes of code values y [..., D] as bytes [..., D * bits / 8]."""
    if bits == 8:
        return y.to(torch.float8_e4m3fn).view(torch.uint8)
    a = y.abs()
    c = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(y).to(torch.uint8)
    return c[..., ::2] | (c[..., 1::2] << 4)


def _pack(case, K, V):
    """Records [b][h][n][bytes] of K and V rows."""
    rec = torch.zeros(*K.shape[:3], _record(case)[2], dtype=torch.uint8, device=K.device)
    at, scales = 0, _record(case)[0] + _record(case)[1]
    for x, bits, place in ((K, case["kbits"], 0), (V, case["vbits"], 4)):
        y, s = _quantized(x, bits)
        codes = _codes(y.reshape(x.shape), bits)
        rec[..., at:at + codes.shape[-1]] = codes
        rec[..., scales + place:scales + place + 4] = (s[..., 0] + 127).to(torch.uint8)
        at += codes.shape[-1]
    return rec


def _values(codes, scales, bits):
    """The values of code bytes [..., D * bits / 8] with scale bytes [..., 4], in 32 bits."""
    c = codes.int()
    if bits == 4:
        c = torch.stack((c & 15, c >> 4), -1).flatten(-2)
    sign, e, m = c >> (bits - 1), (c >> (3 if bits == 8 else 1)) & (15 if bits == 8 else 3), c & (7 if bits == 8 else 1)
    mant, bias = (3, 7) if bits == 8 else (1, 1)
    y = (m + torch.where(e > 0, 1 << mant, 0)).float() * _pow2(e.clamp(min=1) - bias - mant)
    y = torch.where(sign > 0, -y, y).reshape(*codes.shape[:-1], D // BLOCK, BLOCK)
    return (y * _pow2(scales.int() - 127)[..., None]).reshape(*codes.shape[:-1], D)


def _unpack(case, rec):
    kb, vb, _ = _record(case)
    return (_values(rec[..., :kb], rec[..., kb + vb:kb + vb + 4], case["kbits"]),
            _values(rec[..., kb:kb + vb], rec[..., kb + vb + 4:kb + vb + 8], case["vbits"]))


def _attention(q, K, V, visible):
    """softmax(SCALE q K^T) V over the visible pairs in the inputs' precision; 0 where a row sees nothing."""
    s = torch.matmul(q, K.transpose(-1, -2).contiguous()) * SCALE
    s = torch.where(visible, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, V) / torch.where(total > 0, total, 1.0)


def _tree_visible(st, n):
    """Which of n cached rows and t drafts the t drafts see: [b][1][1][t][n + t]."""
    case = st["case"]
    b, t = case["batch"], case["t"]
    at = torch.arange(n, device="cuda")
    lens = st["lens"][:, None, None] if st["lens"] is not None else n
    cached = (at < lens).expand(b, t, n) if st["lens"] is not None else (at < n).expand(b, t, n)
    drafts = (st["mask"][:, :, None] >> torch.arange(t, device="cuda")) & 1 > 0
    return torch.cat((cached, drafts), 2)[:, None, None]


def _sink_visible(st):
    """Which rows the new tokens see [b][1][1][t][n], and which new tokens there are [b][1][t][1]."""
    case = st["case"]
    b, n, t = case["batch"], case["n"], case["t"]
    start = st["starts"][:, None] if st["starts"] is not None else torch.full((b, 1), n - t, device="cuda")
    p = (start + torch.arange(t, device="cuda"))[:, :, None]
    j = torch.arange(n, device="cuda")
    visible = (j <= p) & ((j < case["sink"]) | (j > p - case["window"]))
    count = st["counts"][:, None] if st["counts"] is not None else torch.full((b, 1), t, device="cuda")
    return visible[:, None, None], (torch.arange(t, device="cuda") < count)[:, None, :, None]


def _listed_rows(st, dtype):
    """(K, V, visible) of the rows that each query head lists, and of the window's: [b][h][g][rows][D]."""
    case = st["case"]
    b, h, g, n, k = (case[x] for x in ("batch", "hkv", "g", "n", "k"))
    idx = st["idx"].long().reshape(b, h, g * k)
    rec = st["rec"].to("cuda", non_blocking=True)
    first = st["win"][1] if "win" in st else 0
    rows = torch.gather(rec, 2, (idx.clamp(min=0) + first)[..., None].expand(-1, -1, -1, rec.shape[3]))
    K, V = (x.to(dtype).reshape(b, h, g, k, D) for x in _unpack(case, rows))
    seen = (idx >= 0).reshape(b, h, g, 1, k)
    if "win" in st:
        sink, _, begin, end = st["win"]
        r = torch.arange(sink + end - begin, device="cuda")
        slot = torch.where(r < sink, r, sink + (begin + r - 2 * sink) % (st["K_win"].shape[2] - sink))
        Kw, Vw = (x[:, :, None, slot].to(dtype).expand(-1, -1, g, -1, -1) for x in (st["K_win"], st["V_win"]))
        K, V = torch.cat((Kw, K), 3), torch.cat((Vw, V), 3)
        seen = torch.cat((seen.new_ones(b, h, g, 1, len(r)), seen), 4)
    return K, V, seen


def _plain(st):
    case = st["case"]
    b, h, g, n, t, op = (case[x] for x in ("batch", "hkv", "g", "n", "t", "op"))
    if op == "quant":
        back = []
        for x, bits in ((st["K"], case["kbits"]), (st["V"], case["vbits"])):
            y, s = _quantized(x, bits)
            back.append((y * _pow2(s)).reshape(x.shape).half())
        return {"K": back[0], "V": back[1]}
    if op in ("sparse", "tiered"):
        K, V, seen = _listed_rows(st, torch.float32)
        return {"out": _attention(st["q"].float().reshape(b, h, g, 1, D), K, V, seen).reshape(b, h * g, D)}
    q = st["q"].float().reshape(b, h, g * t, D)
    K, V = _unpack(case, st["rec"]) if "rec" in st else (st["K"].float(), st["V"].float())
    if op == "tree":
        visible = _tree_visible(st, n).expand(b, h, g, t, n + t).reshape(b, h, g * t, n + t)
        K, V = torch.cat((K, st["K_tree"].float()), 2), torch.cat((V, st["V_tree"].float()), 2)
        return {"out": _attention(q, K, V, visible).reshape(b, h * g, t, D)}
    visible, real = _sink_visible(st)
    o = _attention(q, K, V, visible.expand(b, h, g, t, n).reshape(b, h, g * t, n))
    return {"out": torch.where(real, o.reshape(b, h * g, t, D), 0.0).half()}


# ---------------------------------------------------------------- one pass


def _handles(st):
    """What a serving program makes once: the layer's shape, the cache's handle, a workspace."""
    if "cfg" not in st:
        import paper_2602_07721_amd as pk
        case = st["case"]
        b, n, t, op = (case[x] for x in ("batch", "n", "t", "op"))
        cfg = st["cfg"] = pk.Config(case["hkv"], case["g"], n, pk.rotation_signs(1))
        if "rec" in st:
            st["cache"] = pk.QuantCache(st["rec"], case["kbits"], case["vbits"], host_mapped=op == "tiered")
        if op == "tiered":
            st["window"] = pk.Window(*st["win"])
        if op == "tree":
            st["ws"] = torch.empty(pk.tree_workspace_size(cfg, b, n, t), dtype=torch.uint8, device="cuda")
        if op == "sink":
            size = pk.sink_window_workspace_size(cfg, b, n - t, t, case["sink"], case["window"])
            st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        st["pk"] = pk
    return st["pk"], st["cfg"]


def run(st):
    if not own:
        return _plain(st)
    pk, cfg = _handles(st)
    case = st["case"]
    n, t, op = case["n"], case["t"], case["op"]
    if op == "quant":
        row = st["rows"] if st["rows"] is not None else n - t
        pk.quantize_rows(cfg, st["cache"], st["K"], st["V"], 0, row, t)
        pk.dequantize_rows(cfg, st["cache"], row, t, *st["outs"])
        return {"K": st["outs"][0], "V": st["outs"][1]}
    if op == "sparse":
        pk.quant_attend(cfg, st["q"], st["cache"], st["idx"], SCALE, out=st["out"])
    elif op == "tiered":
        pk.quant_tiered_attend(cfg, st["q"], st["K_win"], st["V_win"], st["cache"], st["idx"], st["window"], SCALE,
                               out=st["out"])
    elif op == "tree" and "cache" in st:
        pk.quant_tree_attend(cfg, st["q"], st["cache"], st["K_tree"], st["V_tree"], n, SCALE, mask=st["mask"],
                             lens=st["lens"], out=st["out"], workspace=st["ws"])
    elif op == "tree":
        pk.tree_attend(cfg, st["q"], st["K"], st["V"], st["K_tree"], st["V_tree"], n, SCALE, mask=st["mask"],
                       lens=st["lens"], out=st["out"], workspace=st["ws"])
    else:
        pk.sink_window_attend(cfg, st["q"], st["K"], st["V"], n - t, case["sink"], case["window"], SCALE,
                              starts=st["starts"], counts=st["counts"], out=st["out"], workspace=st["ws"])
    return {"out": st["out"]}


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    b, h, g, n, t, op = (case[x] for x in ("batch", "hkv", "g", "n", "t", "op"))
    rec = 4 * D if case["kbits"] == 16 else _record(case)[2]
    if op in ("tree", "sink") and case["ragged"]:  # lengths between half and all
        n, t = (n * 3 // 4, t) if op == "tree" or n > t else (max(1, n * 3 // 4), max(1, t * 3 // 4))
        n = max(n, t)
    if op == "quant":  # the rows in, their records, the values out
        return {"bytes": b * h * t * (4 * D + rec + 4 * D), "flops": b * h * t * 2 * D * 4}
    if op in ("sparse", "tiered"):
        k, dense = case["k"], SINK + LOCAL + case["buffered"] if op == "tiered" else 0
        return {"bytes": b * h * (min(g * k, n) * rec + dense * 4 * D) + b * h * g * (k * 4 + 2 * D + 4 * D),
                "flops": b * h * g * (k + dense) * 4 * D}
    if op == "tree":
        return {"bytes": b * h * (n * rec + t * 4 * D) + b * h * g * t * 6 * D + b * t * 8,
                "flops": b * h * g * t * (n + t) * 4 * D}
    first, sink, window = n - t, case["sink"], case["window"]

    def pairs(p):  # sum over positions below p of the rows they see
        near = min(p, window)
        pairs_near = near * (near + 1) // 2 + (p - near) * window
        past = max(0, p - window)  # positions that sinks lie behind the window of
        met = min(past, sink)
        return pairs_near + met * (met + 1) // 2 + (past - met) * sink

    low = max(0, first - window + 1)
    rows = n - low + min(sink, low)
    return {"bytes": b * h * rows * 4 * D + b * h * g * t * 4 * D,
            "flops": b * h * g * (pairs(n) - pairs(first)) * 4 * D}


# ---------------------------------------------------------------- the same in 64 bits


def _nearest(x, bits):
    """x [..., D] by the codes' own values: each block scaled, the nearest value looked up, ties to the even code."""
    if bits == 8:
        grid = [(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127]
        s_min = -15
    else:
        grid, s_min = [0, 0.5, 1, 1.5, 2, 3, 4, 6], -23
    grid = torch.tensor(grid, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    x = x.double().reshape(*x.shape[:-1], D // BLOCK, BLOCK)
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.full_like(amax, 2.0 ** s_min)
    for _ in range(40):
        scale = torch.where(amax > grid[-1] * scale, 2 * scale, scale)
    a = x.abs() / scale
    c = torch.bucketize(a, middle)
    c += ((c & 1) == 1) & (a == middle[c.clamp(max=len(middle) - 1)]) & (c < len(middle))
    v = grid[c] * scale
    v = torch.where(v > 65504, grid[(c - 1).clamp(min=0)] * scale, v)
    return torch.where(x < 0, -v, v).reshape(*x.shape[:-2], D)


def _row_of(st, kind):
    """K or V rows of a float16 or quantised cache, by a table of the codes' values."""
    case = st["case"]
    if "rec" not in st:
        return st[kind].double()
    kb, vb, _ = _record(case)
    bits, first, place = (case["kbits"], 0, 0) if kind == "K" else (case["vbits"], kb, 4)
    rec = st["rec"].to("cuda")
    codes = rec[..., first:first + D * bits // 8].long()
    if bits == 4:
        codes = torch.stack((codes % 16, codes // 16), -1).flatten(-2)
        half = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    else:
        half = [(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)]
    table = torch.tensor(half + [-v for v in half], dtype=torch.float64, device="cuda")
    two = torch.tensor([2.0 ** (v - 127) for v in range(256)], dtype=torch.float64, device="cuda")
    scale = two[rec[..., kb + vb + place:kb + vb + place + 4].long()].repeat_interleave(BLOCK, -1)
    return table[codes] * scale


def exact(case, seed):
    st = prepare(case, seed)
    b, h, g, n, t, op = (case[x] for x in ("batch", "hkv", "g", "n", "t", "op"))
    if op == "quant":
        return {"K": _nearest(st["K"], case["kbits"]), "V": _nearest(st["V"], case["vbits"])}
    K, V = _row_of(st, "K"), _row_of(st, "V")
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for i in range(b):
        for j in range(h):
            for r in range(j * g, (j + 1) * g):
                if op in ("sparse", "tiered"):
                    rows = st["idx"][i, r].long()
                    rows = rows[rows >= 0] + (st["win"][1] if op == "tiered" else 0)
                    k, v = K[i, j, rows], V[i, j, rows]
                    if op == "tiered":
                        sink, _, begin, end = st["win"]
                        ring = st["K_win"].shape[2] - sink
                        slots = list(range(sink)) + [sink + (x - sink) % ring for x in range(begin, end)]
                        k = torch.cat((k, st["K_win"][i, j, slots].double()))
                        v = torch.cat((v, st["V_win"][i, j, slots].double()))
                    if len(k):
                        out[i, r] = torch.softmax(k @ st["q"][i, r].double() * SCALE, 0) @ v
                elif op == "tree":
                    m = n if st["lens"] is None else int(st["lens"][i])
                    s = st["q"][i, r].double() @ torch.cat((K[i, j, :m], st["K_tree"][i, j].double())).T * SCALE
                    bit = (st["mask"][i][:, None] >> torch.arange(t, device="cuda")) % 2 == 0
                    s[:, m:][bit] = -math.inf
                    out[i, r] = torch.softmax(s, 1) @ torch.cat((V[i, j, :m], st["V_tree"][i, j].double()))
                else:
                    first = n - t if st["starts"] is None else int(st["starts"][i])
                    real = t if st["counts"] is None else int(st["counts"][i])
                    p = torch.arange(first, first + real, device="cuda")[:, None]
                    j_ = torch.arange(first + real, device="cuda")
                    s = st["q"][i, r, :real].double() @ K[i, j, :first + real].T * SCALE
                    hidden = (j_ > p) | ((j_ >= case["sink"]) & (p - j_ >= case["window"]))
                    out[i, r, :real] = torch.softmax(s.masked_fill(hidden, -math.inf), 1) @ V[i, j, :first + real]
    return {"out": out}
