"""What the operators around the cache are measured on: the rotation that fills it (kvr_rotate), the attention of a
prompt over it (kvr_attend_prompt) and the attention of one new token over its pages (kvr_attend_paged).

A case is one call on one layer. Sizes are those of the named workloads (2k summarisation prompts, 32k and 131k
documents, 32 query heads on 8 key heads, 64 on 8, 32 on 32) or generic ones between and around them. `run` computes
a call in elementary torch operations, or, where `own` is set, makes it through the framework's binding.
"""
import math

import torch

own = False

D = 128
EPS = 1e-6
THETA = 1e6          # of the rotation's frequencies


def _case(kind, context, batch, q_heads, kv_heads, *, new=0, ragged=False, dtype="bf16", page=64, window=0, sink=0,
          scores=False, norm=True, rot=128, style="halves", name=None):
    """context: tokens of the longest sequence, the new ones among them. new: new tokens of a sequence (0: all of
    them, a whole prompt). ragged: the other sequences are shorter, the last of three or more is an empty row of the
    batch. page: tokens a page, 0 for one dense cache."""
    c = dict(kind=kind, context=context, batch=batch, q_heads=q_heads, kv_heads=kv_heads, new=new, ragged=ragged,
             dtype=dtype, page=page, window=window, sink=sink, scores=scores, norm=norm, rot=rot, style=style)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one request decodes: its new token's projections become q and the key for kvr_step_update, all latency
        _case("rotate", 32768, 1, 32, 8, new=1, page=0, name="rotate-1"),
        # four prompts of 8k: rows of a fused projection, keys and values go to the pages
        _case("rotate", 8192, 4, 32, 8, name="rotate-4x8k"),
        # prompts of any length in float32, neighbouring channels paired, a quarter of the channels rotated, no norms
        _case("rotate", 2011, 5, 16, 8, ragged=True, dtype="f32", page=16, norm=False, rot=32, style="pairs",
              name="rotate-ragged-f32"),
        # one short chat: latency
        _case("paged", 1000, 1, 32, 8, new=1, page=16, name="paged-1k"),
        # the throughput configuration: 16 long-document requests together, with the scores that selection reads
        _case("paged", 32768, 16, 32, 8, new=1, scores=True, name="paged-16x32k-scores"),
        # one request over the longest context: few heads, so the cache's length has to be shared out
        _case("paged", 131072, 1, 32, 8, new=1, name="paged-131k"),
        # requests of all lengths under a window with four first tokens, 8 query heads a key head, small pages
        _case("paged", 40009, 48, 64, 8, new=1, ragged=True, page=16, window=4096, sink=4, name="paged-window-ragged"),
        # two prompts of 8k, dense cache, causal
        _case("prompt", 8192, 2, 32, 8, page=0, name="prompt-2x8k"),
        # four summarisation-length prompts with the scores that their compression starts from
        _case("prompt", 2048, 4, 32, 8, page=0, scores=True, name="prompt-4x2k-scores"),
        # a long document under a window with four first tokens
        _case("prompt", 32768, 1, 32, 8, window=4096, sink=4, name="prompt-32k-window"),
        # a short turn after a long context: few rows, much cache
        _case("prompt", 65519, 2, 32, 8, new=48, page=32, name="prompt-48-on-64k"),
        # short prompts of any length in float32, one key head a query head, pages of an odd size
        _case("prompt", 333, 4, 8, 8, ragged=True, dtype="f32", page=24, scores=True, name="prompt-ragged-f32"),
    ]


def draw(rng):
    def log(a, b):
        return int(math.exp(rng.uniform(math.log(a), math.log(b + 1))))

    kind = rng.choice(["rotate", "paged", "prompt"])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 32), (16, 8), (64, 8), (8, 2)])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    common = dict(ragged=rng.random() < 0.5, dtype=dtype, page=rng.choice([0, 16, 16, 24, 64, 128, 256]))
    window, sink = rng.choice([(0, 0), (0, 0), (log(16, 8192), rng.choice([0, 1, 4, 4, 16, 100]))])
    if kind == "rotate":
        one = rng.random() < 0.5
        context = log(1, 8192)
        batch = min(log(1, 64), max(1, (4 << 20) // (context * (q_heads + 2 * kv_heads))))
        rot = rng.choice([128, 128, 64, 32, 2, 0])
        return _case(kind, context, log(1, 128) if one else batch, q_heads, kv_heads, new=1 if one else 0,
                     norm=rng.random() < 0.6, rot=rot, style=rng.choice(["halves", "halves", "pairs"]), **common)
    if kind == "paged":
        context = log(1, 131072)
        batch = min(log(1, 64), max(1, (2 << 20) // (context * kv_heads)))
        return _case(kind, context, batch, q_heads, kv_heads, new=1, window=window, sink=sink,
                     scores=rng.random() < 0.5, **common)
    long_context = rng.random() < 0.3
    context = log(1, 65536 if long_context else 2048 if dtype == "f32" else 8192)
    new = log(1, 128) if long_context else rng.choice([0, 0, 0, log(1, 512)])
    batch = min(log(1, 8), max(1, (1 << 24) // (context * (min(new, context) or context) * q_heads // 32 + 1)))
    return _case(kind, context, batch, q_heads, kv_heads, new=new, window=window, sink=sink,
                 scores=rng.random() < 0.5, **common)


# ---------------------------------------------------------------------------
def lengths(c):
    """Tokens (new ones included) and new tokens of each sequence."""
    n = [c["context"]] * c["batch"]
    if c["ragged"]:
        n = [max(1, int(c["context"] * ((1 - 0.6180339887498949 * b) % 1.0 or 1.0))) for b in range(c["batch"])]
        if c["batch"] >= 3:
            n[-1] = 0
    return n, [min(c["new"], x) if c["new"] else x for x in n]


def _spans(c):
    """Per sequence: (first row of its new tokens, new tokens, tokens)."""
    n, new = lengths(c)
    if c["new"] == 1 and c["kind"] != "prompt":      # one row per sequence, an empty one's too
        new = [1] * c["batch"]
    at, out = 0, []
    for x, y in zip(n, new):
        out.append((at, y, x))
        at += y
    return out, at


def _start(pos, c):
    """First token that the window of a query at `pos` leaves visible."""
    return max(0, pos - c["window"] + 1) if c["window"] else 0


def _pairs_seen(c):
    """(query, key) pairs, and keys that some query sees, over all sequences."""
    pairs = keys = 0
    for _, y, x in _spans(c)[0]:
        if x == 0 or y == 0:
            continue
        for t in range(y):
            p = x - y + t
            lo = _start(p, c)
            pairs += p + 1 - lo + min(c["sink"], lo)
        lo = _start(x - y, c)
        keys += x - lo + min(c["sink"], lo)
    return pairs, keys


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _gen(seed, *ids):
    s = seed
    for i in ids:
        s = (s * 1000003 + i + 1) % (1 << 62)
    return torch.Generator(device="cuda").manual_seed(s)


def prepare(case, seed):
    c = case
    g, dt = _gen(seed, 7), _dtype(c)
    B, Hq, Hkv = c["batch"], c["q_heads"], c["kv_heads"]
    spans, rows = _spans(c)
    n = [x for _, _, x in spans]
    s = {"case": c, "spans": spans, "rows": rows, "table": None, "ps": 0}
    s["n_ctx"] = torch.tensor(n, dtype=torch.int32, device="cuda")
    s["q_start"] = None
    if not (c["new"] == 1 and c["kind"] != "prompt"):
        s["q_start"] = torch.tensor([a for a, _, _ in spans] + [rows], dtype=torch.int32, device="cuda")

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    # the cache: pages in no order, or one row of pages per sequence
    cap = max(1, c["context"])
    ps = c["page"] or cap
    each = -(-cap // ps)
    store = c["kind"] == "rotate" and not (c["new"] == 1 and c["page"] == 0)
    if c["kind"] != "rotate" or store:
        n_pages = B * each
        make = (lambda *sh: torch.zeros(sh, device="cuda", dtype=dt)) if store else normal
        s["k_pool"], s["v_pool"] = make(n_pages, Hkv, ps, D), make(n_pages, Hkv, ps, D)
        s["ps"] = ps
        order = torch.arange(n_pages, device="cuda")
        if c["page"]:
            order = torch.randperm(n_pages, generator=g, device="cuda")
            s["table"] = order.to(torch.int32).view(B, each).contiguous()
        s["pages"] = order.view(B, each)
    if c["kind"] == "rotate":
        fused = normal(rows, Hq + 2 * Hkv, D)         # rows of one projection: the queries, then keys, then values
        s["q"], s["k"], s["v"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        s["wq"] = s["wk"] = None
        if c["norm"]:
            s["wq"], s["wk"] = normal(D) * 0.2 + 1, normal(D) * 0.2 + 1
        half = c["rot"] // 2
        s["inv_freq"] = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(half, 1))
        s["q_out"] = torch.empty(rows, Hq, D, dtype=dt, device="cuda")
        s["k_out"] = None if store else torch.empty(rows, Hkv, D, dtype=dt, device="cuda")
    else:
        # normal queries and keys, and a first token that most heads look at, as trained models have it
        s["q"] = normal(rows, Hq, D)
        u = torch.randn((Hkv, D), generator=g, device="cuda")
        u = torch.nn.functional.normalize(u, dim=-1)
        s["q"] += (2 * u).to(dt).repeat_interleave(Hq // Hkv, dim=0)
        s["k_pool"][s["pages"][:, 0], :, 0] = (20 * u).to(dt)
        s["scores0"] = None
        if c["scores"] and c["kind"] == "paged":      # what earlier tokens left
            s["scores0"] = torch.randn((B, Hkv, cap), generator=g, device="cuda").exp_()
            s["scores"] = torch.empty_like(s["scores0"])
        s["cap"] = cap
    if own:
        _prepare_own(s)
    return s


# ---------------------------------------------------------------------------
# the framework's calls
def _prepare_own(s):
    from paper_2512_17917_amd import binding as kvr
    c = s["case"]
    s["kvr"] = kvr
    s["desc"] = kvr.make_desc(c["batch"], c["q_heads"], c["kv_heads"], 1, 1, _dtype(c))
    s["kv"] = kvr.make_pages(s["desc"], s["k_pool"], s["v_pool"], s["table"]) if "k_pool" in s else None
    if c["kind"] == "rotate":
        s["rot"] = kvr.make_rotation(s["desc"], s["inv_freq"] if c["rot"] else None, q_weight=s["wq"],
                                     k_weight=s["wk"], eps=EPS, pairs=c["style"] == "pairs")
        return
    s["out"] = torch.empty_like(s["q"])
    if c["kind"] == "paged":
        n = kvr.kvr_attend_paged_workspace_size(s["desc"], s["kv"], c["window"], c["sink"], c["scores"])
    else:
        n = kvr.kvr_attend_prompt_workspace_size(s["desc"], s["rows"], s["kv"], c["window"], c["sink"], c["scores"])
    s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")


def _run_own(s):
    c, kvr = s["case"], s["kvr"]
    if c["kind"] == "rotate":
        kvr.kvr_rotate(s["desc"], s["rot"], s["q"], s["k"], s["v"], s["rows"], s["q_start"], s["n_ctx"], s["q_out"],
                       s["k_out"], s["kv"])
        return [s["q_out"]] + ([s["k_out"]] if s["k_out"] is not None else [s["k_pool"], s["v_pool"]])
    scores = _scores_before(s)
    if c["kind"] == "paged":
        kvr.kvr_attend_paged(s["desc"], s["q"], s["n_ctx"], s["kv"], c["window"], c["sink"], s["out"], scores, s["cap"],
                             s["ws"])
    else:
        kvr.kvr_attend_prompt(s["desc"], s["q"], s["rows"], s["q_start"], s["n_ctx"], s["kv"], c["window"], c["sink"],
                              s["out"], scores, s["cap"], s["ws"])
    return [s["out"]] if scores is None else [s["out"], scores]


def _scores_before(s):
    """The cumulated scores that the call adds to: what earlier tokens left, or zeros for a prompt."""
    c = s["case"]
    if not c["scores"]:
        return None
    if s["scores0"] is not None:
        return s["scores"].copy_(s["scores0"])
    return torch.zeros((c["batch"], c["kv_heads"], s["cap"]), device="cuda")


# ---------------------------------------------------------------------------
# the plain forms
def _turned(x, w, pos, inv_freq, pairs):
    """Norm and rotation of rows x [rows, heads, D] at positions pos."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    half = inv_freq.numel()
    if half:
        angle = pos.double()[:, None] * inv_freq      # far positions need the 64 bits
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        head, rest = x[..., :2 * half], x[..., 2 * half:]
        a, b = (head[..., 0::2], head[..., 1::2]) if pairs else (head[..., :half], head[..., half:])
        ra, rb = a * cos - b * sin, b * cos + a * sin
        head = torch.stack([ra, rb], -1).flatten(-2) if pairs else torch.cat([ra, rb], -1)
        x = torch.cat([head, rest], -1)
    return x


def _run_rotate(s):
    c, dt = s["case"], _dtype(s["case"])
    if s["q_start"] is None:
        seq = torch.arange(c["batch"], device="cuda")
        pos = s["n_ctx"].long() - 1
    else:
        new = (s["q_start"][1:] - s["q_start"][:-1]).long()
        seq = torch.repeat_interleave(torch.arange(c["batch"], device="cuda"), new, output_size=s["rows"])
        first = s["n_ctx"].long() - new - s["q_start"][:-1]
        pos = first[seq] + torch.arange(s["rows"], device="cuda")
    pairs = c["style"] == "pairs"
    q = _turned(s["q"], s["wq"], pos, s["inv_freq"], pairs).to(dt)
    k = _turned(s["k"], s["wk"], pos, s["inv_freq"], pairs).to(dt)
    if s["k_out"] is not None:
        return [q, k]
    if c["ragged"]:                                    # a row of an empty sequence has no place
        keep = (pos >= 0).nonzero()[:, 0]
        seq, pos, k, v = seq[keep], pos[keep], k[keep], s["v"][keep]
    else:
        v = s["v"]
    page, row = s["pages"][seq, pos // s["ps"]], pos % s["ps"]
    s["k_pool"][page, :, row] = k
    s["v_pool"][page, :, row] = v
    return [q, s["k_pool"], s["v_pool"]]


def _tokens(s, b, lo, hi):
    """Keys and values [Hkv, hi - lo, D] of tokens lo .. hi-1 of sequence b, in float32."""
    ps = s["ps"]
    p0, p1 = lo // ps, -(-hi // ps)
    pages = s["pages"][b, p0:p1]
    out = []
    for pool in (s["k_pool"], s["v_pool"]):
        x = pool[pages].transpose(0, 1).reshape(pool.shape[1], (p1 - p0) * ps, D)
        out.append(x[:, lo - p0 * ps:hi - p0 * ps].float())
    return out


def _run_attend(s):
    """Sequence by sequence, and blocks of queries that share a range of keys."""
    c = s["case"]
    Hq, Hkv = c["q_heads"], c["kv_heads"]
    G = Hq // Hkv
    out = torch.zeros(s["rows"], Hq, D, dtype=_dtype(c), device="cuda")
    scores = _scores_before(s)
    step = max(1, min(512, (1 << 28) // (Hkv * G * c["context"])))
    for b, (r0, y, x) in enumerate(s["spans"]):
        if x == 0:
            continue
        for t0 in range(0, y, step):
            t1 = min(t0 + step, y)
            p0, p1 = x - y + t0, x - y + t1 - 1
            lo = _start(p0, c)
            first = min(c["sink"], lo)
            k, v = _tokens(s, b, lo, p1 + 1)
            at = torch.arange(lo, p1 + 1, device="cuda")
            if first:
                ks, vs = _tokens(s, b, 0, first)
                k, v = torch.cat([ks, k], 1), torch.cat([vs, v], 1)
                at = torch.cat([torch.arange(first, device="cuda"), at])
            q = s["q"][r0 + t0:r0 + t1].float().view(t1 - t0, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
            w = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1 / math.sqrt(D))
            w = w.view(Hkv, G, t1 - t0, -1)
            if y > 1:
                p = torch.arange(p0, p1 + 1, device="cuda")[:, None]
                seen = at <= p
                if c["window"]:
                    seen &= (at > p - c["window"]) | (at < c["sink"])
                w = w.masked_fill(~seen, -math.inf)
            w = (w - w.amax(-1, keepdim=True)).exp()
            w = w / w.sum(-1, keepdim=True)
            if scores is not None:
                scores[b].index_add_(1, at, w.sum((1, 2)))
            o = torch.matmul(w.view(Hkv, G * (t1 - t0), -1), v)
            out[r0 + t0:r0 + t1] = o.view(Hkv, G, t1 - t0, D).permute(2, 0, 1, 3).reshape(t1 - t0, Hq, D)
    return [out] if scores is None else [out, scores]


def run(state):
    if own:
        return _run_own(state)
    return _run_rotate(state) if state["case"]["kind"] == "rotate" else _run_attend(state)


# ---------------------------------------------------------------------------
def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    spans, rows = _spans(c)
    Hq, Hkv = c["q_heads"], c["kv_heads"]
    if c["kind"] == "rotate":        # every row of q, k (and v, where it goes to the pages) read and written
        store = not (c["new"] == 1 and c["page"] == 0)
        n = rows * (Hq + Hkv * (2 if store else 1)) * D
        turned = rows * (Hq + Hkv)
        return {"bytes": 2 * n * e, "flops": turned * ((4 * D if c["norm"] else 0) + 3 * c["rot"])}
    pairs, keys = _pairs_seen(c)     # rows of q and out, seen keys and values, scores of the seen read and written
    n_bytes = 2 * rows * Hq * D * e + 2 * keys * Hkv * D * e + (8 * keys * Hkv if c["scores"] else 0)
    return {"bytes": n_bytes, "flops": pairs * Hq * D * (6 if c["scores"] and c["kind"] == "prompt" else 4)}


# ---------------------------------------------------------------------------
def exact(case, seed):
    """In 64 bits from the definition: row by row of the projections, or head by head of the attention."""
    s = prepare(case, seed)
    return _exact_rotate(s) if case["kind"] == "rotate" else _exact_attend(s)


def _exact_rotate(s):
    c = s["case"]
    half = c["rot"] // 2
    q_all = torch.empty(s["rows"], c["q_heads"], D, dtype=torch.float64, device="cuda")
    k_all = torch.empty(s["rows"], c["kv_heads"], D, dtype=torch.float64, device="cuda")
    pools = None if s["k_out"] is not None else [s["k_pool"].double(), s["v_pool"].double()]
    for b, (r0, y, x) in enumerate(s["spans"]):
        if y == 0:
            continue
        pos = torch.arange(x - y, x, device="cuda", dtype=torch.float64)
        z = torch.polar(torch.ones_like(pos)[:, None].expand(y, half).contiguous(),
                        torch.outer(pos, s["inv_freq"]))[:, None]
        for src, w, dst in ((s["q"], s["wq"], q_all), (s["k"], s["wk"], k_all)):
            a = src[r0:r0 + y].double()
            if w is not None:
                a = a / (a.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
            if half:
                if c["style"] == "pairs":
                    re, im = a[..., 0:2 * half:2].clone(), a[..., 1:2 * half:2].clone()
                else:
                    re, im = a[..., :half].clone(), a[..., half:2 * half].clone()
                t = torch.complex(re, im) * z
                if c["style"] == "pairs":
                    a[..., 0:2 * half:2], a[..., 1:2 * half:2] = t.real, t.imag
                else:
                    a[..., :half], a[..., half:2 * half] = t.real, t.imag
            dst[r0:r0 + y] = a
        if pools is not None:
            ps = s["ps"]
            for t0 in range(max(0, x - y), x, 1):
                if t0 % ps and t0 != max(0, x - y):
                    continue
                t1 = min(x, (t0 // ps + 1) * ps)       # the rest of one page
                page, i = int(s["pages"][b, t0 // ps]), t0 % ps
                at = r0 + t0 - (x - y)
                pools[0][page, :, i:i + t1 - t0] = k_all[at:at + t1 - t0].transpose(0, 1)
                pools[1][page, :, i:i + t1 - t0] = s["v"][at:at + t1 - t0].transpose(0, 1).double()
    return [q_all, k_all] if pools is None else [q_all] + pools


def _exact_attend(s):
    c = s["case"]
    Hq, Hkv = c["q_heads"], c["kv_heads"]
    G, ps = Hq // Hkv, s["ps"]
    out = torch.zeros(s["rows"], Hq, D, dtype=torch.float64, device="cuda")
    scores = None
    if c["scores"]:
        scores = torch.zeros(c["batch"], Hkv, s["cap"], dtype=torch.float64, device="cuda")
        if s["scores0"] is not None:
            scores += s["scores0"]
    for b, (r0, y, x) in enumerate(s["spans"]):
        if x == 0 or y == 0:
            continue
        j = torch.arange(x, device="cuda")
        page, row = s["pages"][b, j // ps], j % ps
        for h in range(Hkv):
            k, v = s["k_pool"][page, h, row].double(), s["v_pool"][page, h, row].double()
            for g in range(h * G, h * G + G):
                for t0 in range(0, y, 1024):
                    t1 = min(t0 + 1024, y)
                    p = torch.arange(x - y + t0, x - y + t1, device="cuda")[:, None]
                    lo = _start(x - y + t0, c)
                    cols = j[lo:x - y + t1]
                    if lo and c["sink"]:
                        cols = torch.cat([j[:min(c["sink"], lo)], cols])
                    z = s["q"][r0 + t0:r0 + t1, g].double() @ k[cols].T / math.sqrt(D)
                    hidden = cols > p
                    if c["window"]:
                        hidden |= (cols <= p - c["window"]) & (cols >= c["sink"])
                    z[hidden] = -math.inf
                    w = torch.softmax(z, -1)
                    out[r0 + t0:r0 + t1, g] = w @ v[cols]
                    if scores is not None:
                        scores[b, h, cols] += w.sum(0)
    return [out] if scores is None else [out, scores]
