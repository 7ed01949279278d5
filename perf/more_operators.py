"""The operators of a paged K/V cache, as cases to be timed.

plan    pages of the step's new tokens are taken from a stack of free ones: block tables, slots, positions, offsets
rows    a step's queries and keys are normalised for each head and rotated, keys and values written to their slots
attend  attention of the new tokens of many sequences, packed one behind the other, over their pages; scores may be
        capped by a tanh, or get a bias that grows with the distance

A pool of pages is K, V float16 [pages][Hkv][page rows][D].  Row r of sequence b lies in page table[b, r / page rows]; a
slot is page * page rows + row in the page.  New token i of a sequence with `count` new ones and `len` rows, its own
among them, stands at position len - count + i and attends the rows up to that one.

Keys follow the workloads' law: a mean offset per channel, unit scale except 4 outlier channels at 8; values N(0, 1);
half the queries are a cached key plus noise, the others draws from the key law.
"""

import hashlib
import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = D ** -0.5
EPS = 1e-6


def _plan(name, batch, t, n, page, **more):
    """A step of `batch` sequences of up to n rows: t is the size of its token arrays."""
    c = dict(op="plan", batch=batch, t=t, n=n, page=page, chunks=0, ends=0, short=False)
    c.update(more)
    return dict(c, name=name) if name else c


def _rows(name, hkv, g, t, page, **more):
    """t tokens, the last `pad` of them padding; rot: rotated dims."""
    c = dict(op="rows", hkv=hkv, g=g, t=t, page=page, rot=D, norm=True, pairs=False, far=32768, pad=0)
    c.update(more)
    return dict(c, name=name) if name else c


def _attend(name, batch, hkv, g, n, page, **more):
    """Sequences of up to n rows; `chunks` of them have t new tokens, the others one."""
    c = dict(op="attend", batch=batch, hkv=hkv, g=g, n=n, page=page, t=1, chunks=0, ragged=True, cap=0.0, bias=False)
    c.update(more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # A decode step of 64 sequences, a few of which end: latency.
        _plan("plan_step", 64, 64, 8192, 16, ends=3),
        # A full server: 1000 sequences, 40 prompts admitted, 30 that end, and not enough pages for all.
        _plan("plan_burst", 1000, 65536, 16384, 64, chunks=40, ends=30, short=True),
        # A decode step of 32 sequences: latency.
        _rows("rows_step", 8, 4, 32, 16, far=131072),
        # Chunks of a head count that is no power of two, half the dims rotated in neighbouring pairs, no norm.
        _rows("rows_odd", 3, 5, 2501, 48, rot=64, norm=False, pairs=True, pad=37, far=1000000),
        # Prefill of 16384 tokens.
        _rows("rows_prompt", 8, 4, 16384, 64),
        # The smallest step: one sequence of one KV head.
        _attend("step_tiny", 1, 1, 8, 2000, 16, ragged=False),
        # A decode step of 64 sequences of any length, small pages.
        _attend("step_ragged", 64, 8, 4, 16384, 16),
        # Throughput: 8 sequences at 128K tokens.
        _attend("step_8x128k", 8, 8, 4, 131072, 64, ragged=False),
        # Continuous batching: two chunks of prompts next to 30 sequences that decode; pages that end inside tiles.
        _attend("mixed", 32, 8, 4, 20011, 48, t=509, chunks=2),
        # A prompt of 8192 tokens.
        _attend("prompt_8k", 1, 8, 4, 8192, 128, t=8192, chunks=1, ragged=False),
        # Capped scores, prompts of different lengths in chunks.
        _attend("capped_chunks", 3, 4, 2, 8192, 32, t=2048, chunks=3, cap=50.0),
        # Scores with a bias by distance, a decode step of short contexts, 7 heads on a KV head.
        _attend("biased_step", 40, 2, 7, 4096, 16, bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["plan", "plan", "rows", "rows", "rows", "attend", "attend", "attend", "attend", "attend"])
    page = rng.choice([1, 8, 16, 16, 32, 48, 64, 100, 128, 256])
    if op == "plan":
        batch = _log_int(rng, 1, 2000)
        chunks = rng.choice([0, 1, batch // 8, batch // 2]) if rng.random() < 0.6 else 0
        n = _log_int(rng, 16, 16384)
        t = min(65536, batch + chunks * rng.choice([16, 100, 512]))
        return _plan(None, batch, max(t, batch), n, max(page, n // 1024), chunks=min(chunks, batch),
                     ends=rng.randrange(batch // 4 + 1), short=rng.random() < 0.3)
    hkv, g = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
    if op == "rows":
        t = _log_int(rng, 1, max(1, 16384 * 48 // (hkv * (g + 2))))
        return _rows(None, hkv, g, t, page, rot=rng.choice([0, 32, 64, 96, 128, 128]), norm=rng.random() < 0.6,
                     pairs=rng.random() < 0.3, far=rng.choice([4096, 131072, 4000000]), pad=rng.choice([0, 0, t // 5]))
    shape = dict(cap=rng.choice([0.0, 0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.2)
    batch = _log_int(rng, 1, 128)
    n = _log_int(rng, 8, max(8, min(131072, (1 << 23) // (batch * hkv))))
    if rng.random() < 0.5:  # a decode step, or a few tokens of each
        t = rng.choice([1, 1, 1, 2, 4, 9])
        return _attend(None, batch, hkv, g, max(n, t), page, t=t, chunks=batch if t > 1 else 0, **shape)
    chunks = rng.randrange(1, 4)
    batch = max(batch // 4, chunks)
    t = _log_int(rng, 10, 8192)
    n = max(t, min(n, 65536))
    while chunks * hkv * g * t * n > 1 << 30:  # the pairs of the longest prompt listed
        t, n = max(1, t * 3 // 4), max(t, n * 3 // 4)
    return _attend(None, batch, hkv, g, n, page, t=t, chunks=chunks, **shape)


# ---------------------------------------------------------------- inputs


def _seed(case, seed):
    text = ",".join(f"{k}={case[k]}" for k in sorted(case) if k != "name") + f",{seed}"
    return int.from_bytes(hashlib.sha256(text.encode()).digest()[:7], "little")


def _lengths(case):
    """(lens, counts) of an attention case: rows of each sequence, its new tokens among them, and how many are new."""
    rng = random.Random(_seed(case, "lengths"))
    b, n, t = case["batch"], case["n"], case["t"]
    counts = [1] * b
    for i in rng.sample(range(b), case["chunks"]):
        counts[i] = t if not case["ragged"] else rng.randint((t + 1) // 2, t)
    if not case["ragged"]:
        return [n] * b, counts
    return [rng.randint(max(c, n // 16), max(c, n)) for c in counts], counts


def _freqs(rot):
    """Radians a position of the rotated pairs."""
    return torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float32, device="cuda")


def prepare(case, seed):
    s = _seed(case, seed)
    gen, rng = torch.Generator(device="cuda").manual_seed(s), np.random.default_rng(s)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def ints(x):
        return torch.from_numpy(np.asarray(x, dtype=np.int32)).cuda()

    st = dict(case=case)
    page = case["page"]
    if case["op"] == "plan":
        b, t, n = case["batch"], case["t"], case["n"]
        width = -(-n // page) + 2
        lens = rng.integers(1, n + 1, b)
        counts = np.ones(b, dtype=np.int64)
        order = rng.permutation(b)
        new, ends = order[:case["chunks"]], order[case["chunks"]:case["chunks"] + case["ends"]]
        if len(new):  # prompts: sequences that hold nothing yet
            lens[new] = 0
            counts[new] = rng.integers(1, max(2, min(n, (t - b) // len(new) + 1)), len(new))
        counts[ends] = -lens[ends]
        held = -(-lens // page)
        need = (-(-(lens + np.maximum(counts, 0)) // page) - held).sum()
        pages = b * (-(-n // page) + 1)
        spare = int(need) // 2 if case["short"] else pages - int(held.sum())
        perm = rng.permutation(pages)
        table = np.zeros((b, width), dtype=np.int32)
        at = 0
        for i in range(b):
            table[i, :held[i]] = perm[at:at + held[i]]
            at += held[i]
        # Where pages are short, other sequences than this step's hold the rest.
        free = np.zeros(pages, dtype=np.int32)
        free[:spare] = perm[at:at + spare]
        st.update(table=ints(table), free=ints(free), n_free=ints([spare]), lens=ints(lens), counts=ints(counts))
        st["plan"] = {k: ints(np.zeros(m)) for k, m in
                      (("lens", b), ("n_free", 1), ("offsets", b + 1), ("counts", b), ("slots", t), ("positions", t))}
        return st
    hkv, g = case["hkv"], case["g"]
    mu = 0.5 * randn(hkv, D)
    scale = torch.ones(hkv, D, device="cuda")
    scale.scatter_(1, torch.rand(hkv, D, generator=gen, device="cuda").argsort(dim=1)[:, :4], 8.0)
    if case["op"] == "rows":
        t, hq = case["t"], hkv * g
        # One product's output: the queries', keys' and values' columns of a token next to each other.
        x = randn(t, hq + 2 * hkv, D)
        x[:, hq:hq + hkv] = x[:, hq:hq + hkv] * scale + mu
        x = x.half()
        st["q"], st["k"], st["v"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        pages = -(-t // page) + 3
        slots = rng.permutation(pages * page)[:t]
        slots[t - case["pad"]:] = -1
        # Sequences of their own: positions run on from a far one.
        first = rng.integers(0, max(1, case["far"] - t))
        st["slots"], st["positions"] = ints(slots), ints(first + np.arange(t))
        st["freqs"] = _freqs(case["rot"]) if case["rot"] else None
        st["q_weight"], st["k_weight"] = ((1 + 0.1 * randn(D), 1 + 0.1 * randn(D)) if case["norm"] else (None, None))
        st["q_out"] = torch.zeros(t, hq, D, dtype=torch.float16, device="cuda")
        st["K"], st["V"] = (randn(pages, hkv, page, D).half() for _ in range(2))
        return st
    lens, counts = _lengths(case)
    held = [-(-m // page) for m in lens]
    width = max(held) + 1
    pages = sum(held) + 1
    perm = rng.permutation(pages).astype(np.int32)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for i, m in enumerate(held):
        table[i, :m] = perm[at:at + m]
        at += m
    K = torch.empty(pages, hkv, page, D, dtype=torch.float16, device="cuda")
    V = torch.empty_like(K)
    step = max(1, (1 << 27) // (hkv * page * D))
    for i in range(0, pages, step):
        m = min(step, pages - i)
        K[i:i + m] = randn(m, hkv, page, D).mul_(scale[:, None]).add_(mu[:, None]).half()
        V[i:i + m] = randn(m, hkv, page, D).half()
    total = sum(counts)
    q = (mu[:, None] + scale[:, None] * randn(total, hkv, g, D))
    rows = torch.randint(0, pages * page, (total,), generator=gen, device="cuda")
    needle = K[rows // page, :, rows % page].float()[:, :, None] + 0.1 * randn(total, hkv, g, D)
    q[:, :, ::2] = needle[:, :, ::2]
    st["q"] = q.reshape(total, hkv * g, D).half()
    st["K"], st["V"], st["table"], st["lens"] = K, V, ints(table), ints(lens)
    st["offsets"] = ints(np.concatenate(([0], np.cumsum(counts))))
    # A scheduler knows its sequences' lengths on the host as well: those with one new token, and the others.
    st["host"] = (lens, counts)
    st["groups"] = []
    for some in ([i for i, m in enumerate(counts) if m == 1], [i for i, m in enumerate(counts) if m > 1]):
        st["groups"].append((ints(some).long(), max(lens[i] for i in some), max(counts[i] for i in some)) if some else None)
    st["slopes"] = torch.tensor([2.0 ** (-8 * (i + 1) / (hkv * g)) for i in range(hkv * g)], dtype=torch.float32,
                                device="cuda") if case["bias"] else None
    st["out"] = torch.zeros_like(st["q"])
    return st


# ---------------------------------------------------------------- the plain forms


def _plain_plan(st):
    page = st["case"]["page"]
    table, free, lens, counts, n_free = st["table"], st["free"], st["lens"].long(), st["counts"].long(), st["n_free"].long()
    b, width = table.shape
    t, pages = st["plan"]["slots"].shape[0], free.shape[0]
    new = counts.clamp(min=0)
    ends = new.cumsum(0)
    after = (lens + counts).clamp(min=0)
    old_p, new_p = (lens + page - 1) // page, (after + page - 1) // page
    fits = (after <= width * page) & (ends <= t)
    drop = torch.where(counts < 0, old_p - new_p, 0)
    top = n_free + drop.sum()
    need = torch.where((counts > 0) & fits, new_p - old_p, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= top))
    j = torch.arange(width, device="cuda")
    dropped = (counts < 0)[:, None] & (j >= new_p[:, None]) & (j < old_p[:, None])
    i = (drop.cumsum(0) - drop - new_p)[:, None] + j
    more = torch.cat((free, free[:1]))
    more.scatter_(0, torch.where(dropped, top - 1 - i, pages).reshape(-1), table.reshape(-1))
    free.copy_(more[:pages])
    taken = (ok & (counts > 0))[:, None] & (j >= old_p[:, None]) & (j < new_p[:, None])
    i = (upto - need - old_p)[:, None] + j
    table.copy_(torch.where(taken, free[(top - 1 - i).clamp(0, pages - 1)], table))
    granted = torch.where(ok, new, 0)
    at = torch.arange(t, device="cuda")
    seq = torch.searchsorted(ends, at, right=True)
    real = seq < b
    seq = seq.clamp(max=b - 1)
    real &= granted[seq] > 0
    pos = lens[seq] + at - (ends - new)[seq]
    slot = table[seq, (pos // page).clamp(0, width - 1)] * page + pos % page
    return {"table": table, "free": free, "lens": torch.where(ok | (counts < 0), after, lens).int(),
            "n_free": (top - torch.where(ok, need, 0).sum()).int(),
            "offsets": torch.cat((ends[:1] * 0, ends)).clamp(max=t).int(), "counts": granted.int(),
            "slots": torch.where(real, slot, -1).int(), "positions": torch.where(real, pos, -1).int()}


def _plain_rows(st):
    case = st["case"]
    rot, page = case["rot"], case["page"]
    if rot:
        angle = st["positions"].double()[:, None] * st["freqs"].double()
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        if not rot:
            return x
        y = x.clone()
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y

    real = case["t"] - case["pad"]
    slots = st["slots"][:real].long()
    st["q_out"][:real] = turn(st["q"], st["q_weight"])[:real].half()
    st["K"][slots // page, :, slots % page] = turn(st["k"], st["k_weight"])[:real].half()
    st["V"][slots // page, :, slots % page] = st["v"][:real]
    return {"q": st["q_out"], "K": st["K"], "V": st["V"]}


def _attention(st, seqs, n, t, out):
    """The sequences seqs, padded to n rows and t new tokens, into out, whose last row takes the padding."""
    case = st["case"]
    hkv, g, page = case["hkv"], case["g"], case["page"]
    b, pages = seqs.shape[0], -(-n // page)
    lens, begin, count = (x[:, None] for x in (st["lens"][seqs], st["offsets"][seqs], st["offsets"].diff()[seqs]))
    table = st["table"][seqs, :pages].long().clamp(min=0)
    # [b][pages][hkv][page][D] -> [b hkv][n][D]
    K, V = (st[k][table].transpose(1, 2).reshape(b * hkv, pages * page, D)[:, :n].float() for k in ("K", "V"))
    i, j = torch.arange(t, device="cuda"), torch.arange(n, device="cuda")
    rows = torch.where(i < count, begin + i, out.shape[0] - 1)
    q = st["q"][rows.clamp(max=out.shape[0] - 2)].float().reshape(b, t, hkv, g, D).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.reshape(b * hkv, g * t, D), K.transpose(1, 2).contiguous()).reshape(b, hkv, g, t, n) * SCALE
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    far = j - (lens - count + i)[:, :, None]
    if case["bias"]:
        s = s + st["slopes"].reshape(hkv, g, 1, 1) * far[:, None, None]
    s = torch.where((far <= 0)[:, None, None], s, -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    total = p.sum(-1, keepdim=True)
    V = torch.where((j < lens)[:, None, :, None], V.reshape(b, hkv, n, D), 0.0).reshape(b * hkv, n, D)
    o = torch.matmul(p.reshape(b * hkv, g * t, n), V).reshape(b, hkv, g, t, D) / total
    out[rows] = o.permute(0, 3, 1, 2, 4).reshape(b, t, hkv * g, D).half()


def _plain_attend(st):
    out = torch.cat((st["out"], st["out"][:1]))
    singles, chunks = st["groups"]
    if singles is not None:
        _attention(st, *singles, out)
    if chunks is not None:
        _attention(st, *chunks, out)
    return {"out": out[:-1]}


# ---------------------------------------------------------------- one pass


def _handles(st):
    """What a serving program makes once: the layer's shape, the cache's handle, a workspace."""
    if "pk" not in st:
        import paper_2602_07721_amd as pk
        case = st["case"]
        if case["op"] == "plan":
            st["pages"] = pk.PagePlan(**st["plan"])
        else:
            st["cfg"] = pk.Config(case["hkv"], case["g"], 1, pk.rotation_signs(1))
            st["cache"] = pk.PagedCache(st["K"], st["V"])
        if case["op"] == "attend":
            st["most"] = max(st["host"][1])
            size = pk.paged_workspace_size(st["cfg"], case["batch"], st["q"].shape[0], st["most"])
            st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        st["pk"] = pk
    return st["pk"]


def run(st):
    case = st["case"]
    if not own:
        return {"plan": _plain_plan, "rows": _plain_rows, "attend": _plain_attend}[case["op"]](st)
    pk = _handles(st)
    if case["op"] == "plan":
        pk.plan_pages(st["table"], st["free"], st["n_free"], st["lens"], st["counts"], case["page"], plan=st["pages"])
        return dict(st["plan"], table=st["table"], free=st["free"])
    if case["op"] == "rows":
        pk.rotate_rows(st["cfg"], st["cache"], st["q"], st["k"], st["v"], st["positions"], st["slots"], freqs=st["freqs"],
                       q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, pairs=case["pairs"], q_out=st["q_out"])
        return {"q": st["q_out"], "K": st["K"], "V": st["V"]}
    pk.paged_attend(st["cfg"], st["q"], st["cache"], st["table"], st["lens"], st["offsets"], SCALE, max_tokens=st["most"],
                    softcap=case["cap"], slopes=st["slopes"], out=st["out"], workspace=st["ws"])
    return {"out": st["out"]}


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    if case["op"] == "plan":
        b, t = case["batch"], case["t"]
        return {"bytes": b * 20 + t * 8 + t // case["page"] * 8, "flops": b * 8 + t * 4}
    hkv, g = case["hkv"], case["g"]
    if case["op"] == "rows":
        t = case["t"] - case["pad"]
        return {"bytes": t * (hkv * (g + 2) * 4 * D + 8), "flops": t * hkv * (g + 1) * 8 * D}
    lens, counts = _lengths(case)
    pairs = sum(m * n - m * (m - 1) // 2 for n, m in zip(lens, counts))
    return {"bytes": sum(lens) * hkv * 4 * D + sum(counts) * hkv * g * 4 * D + sum(-(-n // case["page"]) for n in lens) * 4,
            "flops": pairs * hkv * g * 4 * D}


# ---------------------------------------------------------------- the same in 64 bits


def _exact_plan(st):
    page = st["case"]["page"]
    table, free, lens, counts = (st[k].cpu().tolist() for k in ("table", "free", "lens", "counts"))
    n_free, t = int(st["n_free"]), len(st["plan"]["slots"])
    dropped = []
    for b, c in enumerate(counts):
        if c < 0:
            keep = -(-max(0, lens[b] + c) // page)
            dropped += table[b][keep:-(-lens[b] // page)]
    stack = free[:n_free] + dropped[::-1]
    free[n_free:len(stack)] = dropped[::-1]
    top = len(stack)
    offsets, granted, after, slots, positions = [0], [], [], [-1] * t, [-1] * t
    wanted, at = 0, 0
    for b, c in enumerate(counts):
        m = max(c, 0)
        total = max(0, lens[b] + c)
        have, need = -(-lens[b] // page), -(-total // page)
        ok = c > 0 and total <= len(table[b]) * page and at + m <= t
        if ok:
            begin, wanted = wanted, wanted + need - have
            ok = need == have or wanted <= top
        if ok:
            for j in range(have, need):
                table[b][j] = stack[top - 1 - begin - (j - have)]
            for i in range(m):
                p = lens[b] + i
                slots[at + i], positions[at + i] = table[b][p // page] * page + p % page, p
        granted.append(m if ok else 0)
        after.append(total if ok or c < 0 else lens[b])
        at += m
        offsets.append(min(at, t))
    used = sum(-(-x // page) for x in after)
    left = int(st["n_free"]) + sum(-(-x // page) for x in lens) - used
    whole = {"table": table, "free": free, "lens": after, "n_free": [left], "offsets": offsets, "counts": granted,
             "slots": slots, "positions": positions}
    return {k: torch.tensor(v, dtype=torch.int32) for k, v in whole.items()}


def _exact_rows(st):
    case = st["case"]
    rot, half, page = case["rot"], case["rot"] // 2, case["page"]
    t = case["t"] - case["pad"]
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + half)
    out = {"q": st["q_out"].double(), "K": st["K"].double(), "V": st["V"].double()}
    for name, w in (("q", st["q_weight"]), ("k", st["k_weight"])):
        x = st[name][:t].double()
        if w is not None:
            x = w.double() * x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS)
        if rot:
            angle = torch.outer(st["positions"][:t].double(), st["freqs"].double())
            z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)[:, None]
            x[..., first], x[..., second] = z.real, z.imag
        if name == "q":
            out["q"][:t] = x
        else:
            slots = st["slots"][:t].long()
            flat = out["K"].transpose(1, 2).reshape(-1, case["hkv"], D)
            flat[slots] = x
            out["K"] = flat.reshape(-1, page, case["hkv"], D).transpose(1, 2)
            flat = out["V"].transpose(1, 2).reshape(-1, case["hkv"], D)
            flat[slots] = st["v"][:t].double()
            out["V"] = flat.reshape(-1, page, case["hkv"], D).transpose(1, 2)
    return out


def _exact_attend(st):
    case = st["case"]
    hkv, g, page = case["hkv"], case["g"], case["page"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    begin = 0
    for b, (n, m) in enumerate(zip(*st["host"])):
        r = torch.arange(n, device="cuda")
        page_of = st["table"][b].long()[r // page]
        p = torch.arange(n - m, n, device="cuda")
        for h in range(hkv):
            k, v = st["K"][page_of, h, r % page].double(), st["V"][page_of, h, r % page].double()
            for x in range(h * g, (h + 1) * g):
                for lo in range(0, m, 4096):
                    pos = p[lo:lo + 4096, None]
                    s = st["q"][begin + lo:begin + min(lo + 4096, m), x].double() @ k.T / math.sqrt(D)
                    if case["cap"] > 0:
                        s = torch.tanh(s / case["cap"]) * case["cap"]
                    if st["slopes"] is not None:
                        s -= st["slopes"][x].double() * (pos - r)
                    out[begin + lo:begin + min(lo + 4096, m), x] = torch.softmax(s.masked_fill(r > pos, -math.inf), 1) @ v
        begin += m
    return {"out": out}


def exact(case, seed):
    st = prepare(case, seed)
    return {"plan": _exact_plan, "rows": _exact_rows, "attend": _exact_attend}[case["op"]](st)
