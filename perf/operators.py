"""The calls that extend a recovered cache with new tokens, as cases to time and compare.

A service that keeps recovered prefixes in 16-token pages continues them: a conversation's next turn, a
run of drafted tokens, one generated token for each row of a batch. Between two adapter updates it makes
these calls of one layer or of the pool:

* ``rotary``: rotary positions on the query and key heads of a batch of rows (``Context.rotary``); with
  ``inverse`` the rotation back, which is the gradient and also lifts cached keys off their positions.
* ``append``: the rows of several requests rotated, their keys and values written into the requests' pages
  (``Context.cache_append``).
* ``attention``: those rows over their requests' cached keys (``Context.chunk_attention``).
* ``fork``, ``compact``, ``release``: pages shared or copied for a second continuation, moved to the pool's
  front, given back (``Context.pages_fork``, ``pages_compact``, ``pages_release``).

Head counts and pools are those of the tiny decoder and of the two Qwen2.5 shapes; page tables are random
permutations of the pool.
"""
import math

import torch

own = False

PAGE = 16
DEV = "cuda:0"

# layers, query heads, kv heads, head dim, rope theta
SHAPES = {"tiny": (4, 4, 2, 64, 1e4), "1.5b": (28, 12, 2, 128, 1e6), "7b": (28, 28, 4, 128, 1e6)}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the next generated token of one conversation: two heads' worth of bytes, launch and latency
        dict(name="rotary-row", kind="rotary", shape="1.5b", tokens=1, rot=64, layout="interleaved", scaling="none", type="fp16", inverse=False, top=16000),
        # the gradient of a long sequence's rotation in fp32, frequencies scaled by bands for a longer context
        dict(name="rotary-16k-inverse", kind="rotary", shape="7b", tokens=16384, rot=128, layout="half", scaling="bands", type="fp32", inverse=True, top=131072),
        # a batch of generated tokens, one a request, far into their caches
        dict(name="append-rows", kind="append", shape="7b", chunks="32x1", keys_min=900, keys_max=15000, rot=128, layout="half", scaling="none"),
        # two prompts' next turns, odd lengths
        dict(name="append-chunks", kind="append", shape="7b", chunks="4096,3001", keys_min=5003, keys_max=16384, rot=128, layout="half", scaling="linear"),
        # one generated token over a short cache: latency
        dict(name="attention-row", kind="attention", shape="tiny", chunks="1", keys_min=300, keys_max=300, window=0),
        # a batch of generated tokens over long caches: bytes
        dict(name="attention-rows", kind="attention", shape="7b", chunks="8x1", keys_min=4000, keys_max=16384, window=0),
        # requests of every kind in one call: a drafted run, single tokens, next turns; local layers' window
        dict(name="attention-ragged", kind="attention", shape="1.5b", chunks="5,1,517,1,130,64", keys_min=700, keys_max=8200, window=2048),
        # the next turn of a long conversation: matrix products
        dict(name="attention-chunk", kind="attention", shape="7b", chunks="4096", keys_min=16384, keys_max=16384, window=0),
        # eight continuations of cached prefixes: whole pages shared, the last one's live slots copied
        dict(name="pages-fork", kind="fork", shape="7b", layers=28, tables=8, tokens_min=1000, tokens_max=4001, free=64, deep=False),
        # a private copy of a long prefix, before its recovery overwrites it
        dict(name="pages-copy", kind="fork", shape="7b", layers=28, tables=1, tokens_min=16379, tokens_max=16379, free=1100, deep=True),
        # a pool that requests left with holes, packed again
        dict(name="pages-compact", kind="compact", shape="1.5b", layers=28, tables=24, tokens_min=300, tokens_max=9000, free=1500),
        # a large pool's ended requests, sharing pages
        dict(name="pages-release", kind="release", shape="tiny", tables=64, tokens_min=2000, tokens_max=16384, free=30000),
    ]


def chunk_lengths(case):
    """"4096,3001" or "32x1"."""
    if "x" in case["chunks"]:
        n, m = case["chunks"].split("x")
        return [int(m)] * int(n)
    return [int(c) for c in case["chunks"].split(",")]


def spread_over(n, a, b):
    """n whole numbers spread geometrically over [a, b], largest first."""
    return [int(round(b * (a / b) ** (i / max(1, n - 1)))) for i in range(n)]


def keys_of(case):
    """Cached keys of each request, its new rows' among them."""
    new = chunk_lengths(case)
    return [max(k, m) for k, m in zip(spread_over(len(new), case["keys_min"], case["keys_max"]), new)]


def table_tokens(case):
    """Tokens of each page table; odd ones among them."""
    return spread_over(case["tables"], case["tokens_min"], case["tokens_max"])


def draw(rng):
    def spread(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    shape = rng.choice(("tiny", "1.5b", "7b"))
    layers, hq, hkv, d, _ = SHAPES[shape]
    layout, scaling = rng.choice(("half", "half", "interleaved")), rng.choice(("none", "none", "linear", "base", "bands"))
    rot = rng.choice((d, d, d // 2, d // 4))
    kind = rng.choice(("rotary", "append", "attention", "attention", "attention", "fork", "compact", "release"))
    if kind == "rotary":
        return dict(kind=kind, shape=shape, tokens=spread(1, 16384), rot=rot, layout=layout, scaling=scaling, type=rng.choice(("bf16", "bf16", "fp16", "fp32")), inverse=rng.random() < 0.4, top=spread(200, 131072))
    if kind in ("append", "attention"):
        n = rng.choice((1, 1, 2, 3, 5, 8, 16, 32, 48))
        room, new = 4096, []  # new rows left
        for _ in range(n):
            m = rng.choice((1, 1, 1, spread(1, 16), spread(2, 4096)))
            new.append(max(1, min(m, room // 2 if len(new) else room)))
            room -= new[-1]
        if rng.random() < 0.3:
            new = [1] * n
        top = 16384 if n <= 4 else 16384 * 4 // n  # the largest listed call reads about as many keys
        a, b = sorted((spread(16, top), spread(16, top)))
        c = dict(kind=kind, shape=shape, chunks=",".join(map(str, new)), keys_min=a, keys_max=b)
        return dict(c, rot=rot, layout=layout, scaling=scaling) if kind == "append" else dict(c, window=rng.choice((0, 0, 0, spread(16, 4096))))
    n = spread(1, 64)
    a, b = sorted((spread(16, 16384 // n + 16), spread(16, 16384 // n + 16)))
    c = dict(kind=kind, shape=shape, tables=n, tokens_min=a, tokens_max=b)
    if kind == "release":
        return dict(c, free=spread(16, 30000))
    free = b // PAGE * n + n + spread(16, 500) if kind == "fork" else spread(16, 500)
    c.update(layers=rng.randint(1, layers), free=free)
    return dict(c, deep=rng.random() < 0.5) if kind == "fork" else c


# ---------------------------------------------------------------------------------------------- inputs
class Draws:
    """Seeded values on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=self.g)

    def ints(self, n, top):
        return torch.randint(0, top, (n,), dtype=torch.int32, device=DEV, generator=self.g)

    def pages(self, n):
        return torch.randperm(n, device=DEV, generator=self.g).to(torch.int32)


def rope_args(case):
    theta = SHAPES[case["shape"]][4]
    a = dict(head_dim=SHAPES[case["shape"]][3], rot_dim=case["rot"], theta=theta, layout=case["layout"], scaling=case["scaling"])
    if case["scaling"] != "none":
        a["factor"] = 4.0
    if case["scaling"] == "bands":
        a.update(low=1.0, high=32.0, original=32768, magnitude=0.1 * math.log(4.0) + 1.0)
    return a


def pages_for(n):
    return (n + PAGE - 1) // PAGE


def prepare(case, seed):
    d = Draws(seed)
    layers, hq, hkv, dim, _ = SHAPES[case["shape"]]
    s = {"case": case, "kind": case["kind"]}
    if case["kind"] == "rotary":
        # q and k as a fused projection leaves them: heads of one row side by side
        n, t = case["tokens"], TYPES[case["type"]]
        x = d.normal((n, hq + hkv, dim), t)
        s.update(q=x[:, :hq], k=x[:, hq:], positions=d.ints(n, case["top"]), q_out=torch.empty_like(x[:, :hq], memory_format=torch.contiguous_format), k_out=torch.empty_like(x[:, hq:], memory_format=torch.contiguous_format))
    elif case["kind"] in ("append", "attention"):
        new, keys = chunk_lengths(case), keys_of(case)
        counts = [pages_for(k) for k in keys]
        perm = d.pages(sum(counts) + 5)
        s.update(new=new, keys=keys, tables=[t.contiguous() for t in perm[: sum(counts)].split(counts)])
        shape = (len(perm), hkv, PAGE, dim)
        s["k_pages"] = d.normal(shape)
        # values share a mean a channel, as a trained layer's do
        s["v_pages"] = (d.normal(shape, torch.float32) + 0.5 * d.normal((hkv, 1, dim), torch.float32)).bfloat16()
        rows = sum(new)
        if case["kind"] == "append":
            qkv = d.normal((rows, hq + 2 * hkv, dim))
            s.update(q=qkv[:, :hq], k=qkv[:, hq : hq + hkv], v=qkv[:, hq + hkv :], q_out=torch.empty(rows, hq, dim, dtype=torch.bfloat16, device=DEV))
        else:
            s.update(q=d.normal((rows, hq, dim)), out=torch.empty(rows, hq, dim, dtype=torch.bfloat16, device=DEV), lse=torch.empty(rows, hq, dtype=torch.float32, device=DEV))
    else:
        tokens = table_tokens(case)
        counts = [pages_for(n) for n in tokens]
        total = sum(counts) + case["free"]
        perm = d.pages(total)
        tables = [t.contiguous() for t in perm[: sum(counts)].split(counts)]
        if case["kind"] != "fork":
            # every other request continues a prefix that it shares with the one before it
            for i in range(1, len(tables), 2):
                shared = min(counts[i], counts[i - 1]) // 2
                tables[i][:shared] = tables[i - 1][:shared]
        every = torch.cat(tables).long()
        refs = torch.zeros(total, dtype=torch.int32, device=DEV).index_add_(0, every, torch.ones_like(every, dtype=torch.int32))
        if case["kind"] == "release":
            refs += d.ints(total, 2)  # held elsewhere too, or free
        new_tables = torch.empty(sum(counts), dtype=torch.int32, device=DEV)
        s.update(tokens=tokens, tables=tables, refs=refs, refs_out=torch.empty_like(refs), new_tables=new_tables, tables_out=list(new_tables.split(counts)))
        if case["kind"] != "release":
            shape = (case["layers"], total, hkv, PAGE, dim)
            s.update(k_pages=d.normal(shape), v_pages=d.normal(shape))
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def frequencies(a, dtype=torch.float64):
    """Radians a position of each pair."""
    rot, theta, s = a["rot_dim"], a["theta"], a.get("factor", 1.0)
    if a["scaling"] == "base":
        theta = theta * s ** (rot / (rot - 2))
    f = theta ** (-torch.arange(0, rot, 2, dtype=dtype, device=DEV) / rot)
    if a["scaling"] == "linear":
        f = f / s
    if a["scaling"] == "bands":
        turns = a["original"] * f / (2 * math.pi)
        keep = ((turns - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
        f = f * keep + f / s * (1 - keep)
    return f


def rotated(x, positions, a, inverse=False):
    """x [rows, heads, dim] at ``positions``: angles in 64 bits, products in 32, rounded once."""
    rot = a["rot_dim"]
    angle = positions.double()[:, None] * frequencies(a)[None]
    mag = a.get("magnitude", 1.0)
    c, n = (angle.cos() * mag).float()[:, None], (angle.sin() * mag * (-1 if inverse else 1)).float()[:, None]
    w = x.float()
    if a["layout"] == "half":
        u, v, rest = w[..., : rot // 2], w[..., rot // 2 : rot], w[..., rot:]
        y = torch.cat((u * c - v * n, v * c + u * n, rest), -1)
    else:
        u, v, rest = w[..., 0:rot:2], w[..., 1:rot:2], w[..., rot:]
        y = torch.cat((torch.stack((u * c - v * n, v * c + u * n), -1).flatten(-2), rest), -1)
    return y.to(x.dtype)


def row_table(s):
    """Request and position of each new row, on the GPU."""
    new = torch.tensor(s["new"], device=DEV)
    pos0 = torch.tensor(s["keys"], device=DEV) - new
    b = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEV), new, output_size=sum(s["new"]))
    i = torch.arange(sum(s["new"]), device=DEV) - (new.cumsum(0) - new)[b]
    return b, pos0[b] + i, i


def padded_tables(s):
    return torch.nn.utils.rnn.pad_sequence(s["tables"], batch_first=True).long()


def plain_append(s):
    a = rope_args(s["case"])
    b, p, _ = row_table(s)
    page, slot = padded_tables(s)[b, p // PAGE], p % PAGE
    s["q_out"].copy_(rotated(s["q"], p, a))
    s["k_pages"][page, :, slot] = rotated(s["k"], p, a)
    s["v_pages"][page, :, slot] = s["v"]
    return s["q_out"], s["k_pages"], s["v_pages"]


def plain_attention(s):
    """Every request padded to the longest: scores, row maxima, weights and their sums in 32 bits."""
    b, p, i = row_table(s)
    hq, dim = s["q"].shape[1:]
    hkv = s["k_pages"].shape[1]
    g, m, window = hq // hkv, max(s["new"]), s["case"]["window"]
    t = padded_tables(s)
    nb, n = t.shape[0], t.shape[1] * PAGE
    keys = torch.tensor(s["keys"], device=DEV)
    k = s["k_pages"][t].float().permute(0, 2, 1, 3, 4).reshape(nb, hkv, n, dim)
    v = s["v_pages"][t].float().permute(0, 2, 1, 3, 4).reshape(nb, hkv, n, dim)
    j = torch.arange(n, device=DEV)
    v = torch.where((j[None] < keys[:, None])[:, None, :, None], v, 0.0)
    q = torch.zeros(nb, m, hq, dim, device=DEV)
    q[b, i] = s["q"].float()
    q = q.view(nb, m, hkv, g, dim).permute(0, 2, 3, 1, 4).reshape(nb, hkv, g * m, dim)
    at = torch.zeros(nb, m, dtype=torch.long, device=DEV)
    at[b, i] = p
    seen = (j <= at[..., None]) & (j < keys[:, None, None])
    if window:
        seen &= j > at[..., None] - window
    z = (q @ k.transpose(-1, -2) * dim**-0.5).view(nb, hkv, g, m, n).masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    z = z.sub_(torch.where(top.isinf(), 0.0, top)).exp_()
    total = z.sum(-1, keepdim=True)
    o = (z.view(nb, hkv, g * m, n) @ v).view(nb, hkv, g, m, dim) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log()).squeeze(-1)
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(nb, m, hq, dim)[b, i])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(nb, m, hq)[b, i])
    return s["out"], s["lse"]


def lowest_free(refs, count):
    """The ``count`` lowest pages that nothing refers to, in order."""
    free = refs == 0
    rank = torch.where(free, free.cumsum(0) - 1, count).clamp(max=count)
    ids = torch.arange(len(refs), device=DEV)
    return torch.zeros(count + 1, dtype=torch.long, device=DEV).scatter_(0, rank, ids)[:count]


def plain_fork(s):
    deep, tokens = s["case"]["deep"], torch.tensor(s["tokens"], device=DEV)
    pages = (tokens + PAGE - 1) // PAGE
    parent = torch.cat(s["tables"]).long()
    f = torch.repeat_interleave(torch.arange(len(pages), device=DEV), pages, output_size=len(parent))
    e = torch.arange(len(parent), device=DEV) - (pages.cumsum(0) - pages)[f]
    live = (tokens[f] - e * PAGE).clamp(max=PAGE)  # live slots of each entry's page
    fresh = torch.ones_like(live, dtype=torch.bool) if deep else live < PAGE
    count = sum(pages_for(n) if deep else (n % PAGE > 0) for n in s["tokens"])
    free = lowest_free(s["refs"], count)
    child = parent.clone()
    at = fresh.nonzero().squeeze(1)
    child[at] = free
    s["refs_out"].copy_(s["refs"])
    s["refs_out"].index_add_(0, child, torch.ones_like(child, dtype=torch.int32))
    src = parent[at]
    keep = (torch.arange(PAGE, device=DEV) < live[at][:, None])[None, :, None, :, None]
    s["k_pages"][:, free] = torch.where(keep, s["k_pages"][:, src], s["k_pages"][:, free])
    s["v_pages"][:, free] = torch.where(keep, s["v_pages"][:, src], s["v_pages"][:, free])
    return child.to(torch.int32), s["refs_out"], s["k_pages"], s["v_pages"]


def plain_compact(s):
    live = s["refs"] > 0
    n = live.sum()
    ids = torch.arange(len(live), device=DEV)
    holes, movers = (~live & (ids < n)).nonzero().squeeze(1), (live & (ids >= n)).nonzero().squeeze(1)
    to = ids.clone()
    to[movers] = holes
    s["refs_out"].copy_(torch.where(ids < n, s["refs"], 0))
    s["refs_out"][holes] = s["refs"][movers]
    s["k_pages"][:, holes] = s["k_pages"][:, movers]
    s["v_pages"][:, holes] = s["v_pages"][:, movers]
    return to[torch.cat(s["tables"]).long()].to(torch.int32), s["refs_out"], s["k_pages"], s["v_pages"]


def plain_release(s):
    every = torch.cat(s["tables"]).long()
    s["refs_out"].copy_(s["refs"])
    s["refs_out"].index_add_(0, every, torch.full_like(every, -1, dtype=torch.int32))
    return s["refs_out"]


# ---------------------------------------------------------------------------------------------- the framework's calls
HELD = {}


def page_tables(s):
    """The tables of one call. The requests that fork, move or end are other ones at every call, and have grown: no
    program has this at hand."""
    import paper_2609_30884_gb300 as crf

    return crf.PageTables(s["tables"], s["tokens"], None if s["kind"] == "release" else s["tables_out"])


def held(s):
    """What a program keeps across its layers and steps: the context, the pool, a step's chunks, a workspace."""
    import paper_2609_30884_gb300 as crf

    if "ctx" not in HELD:
        HELD["ctx"] = crf.Context(0)
    ctx, case, kind = HELD["ctx"], s["case"], s["kind"]
    h = {"ctx": ctx}
    if kind in ("rotary", "append"):
        h["rope"] = crf.Rope(**rope_args(case))
    if kind in ("append", "attention"):
        h["pool"] = crf.KVPool([s["k_pages"]], [s["v_pages"]])
        h["chunks"] = crf.Chunks(s["tables"], s["new"], [k - m for k, m in zip(s["keys"], s["new"])])
    if kind == "attention":
        h["ws"] = ctx.chunk_attention_workspace(h["pool"], h["chunks"], s["q"].shape[1], window=case["window"])
    if kind in ("fork", "compact", "release"):
        h["ws"] = ctx.pages_workspace(len(s["refs"]), page_tables(s))
        if kind != "release":
            h["pool"] = crf.KVPool(list(s["k_pages"]), list(s["v_pages"]))
    return h


def own_run(s):
    if "held" not in s:
        s["held"] = held(s)
    h, kind = s["held"], s["kind"]
    ctx = h["ctx"]
    if kind == "rotary":
        ctx.rotary(h["rope"], s["positions"], s["q"], s["q_out"], k=s["k"], k_out=s["k_out"], inverse=s["case"]["inverse"])
        return s["q_out"], s["k_out"]
    if kind == "append":
        ctx.cache_append(h["pool"], 0, h["chunks"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=h["rope"])
        return s["q_out"], s["k_pages"], s["v_pages"]
    if kind == "attention":
        ctx.chunk_attention(h["pool"], 0, h["chunks"], s["q"], s["out"], h["ws"], lse=s["lse"], window=s["case"]["window"])
        return s["out"], s["lse"]
    if kind == "fork":
        ctx.pages_fork(h["pool"], s["refs"], page_tables(s), h["ws"], refs_out=s["refs_out"], deep=s["case"]["deep"])
        return s["new_tables"], s["refs_out"], s["k_pages"], s["v_pages"]
    if kind == "compact":
        ctx.pages_compact(h["pool"], s["refs"], page_tables(s), h["ws"], refs_out=s["refs_out"])
        return s["new_tables"], s["refs_out"], s["k_pages"], s["v_pages"]
    ctx.pages_release(s["refs"], page_tables(s), h["ws"], refs_out=s["refs_out"])
    return s["refs_out"]


def run(s):
    if own:
        return own_run(s)
    kind = s["kind"]
    if kind == "rotary":
        a, inv = rope_args(s["case"]), s["case"]["inverse"]
        s["q_out"].copy_(rotated(s["q"], s["positions"], a, inv))
        s["k_out"].copy_(rotated(s["k"], s["positions"], a, inv))
        return s["q_out"], s["k_out"]
    return {"append": plain_append, "attention": plain_attention, "fork": plain_fork, "compact": plain_compact, "release": plain_release}[kind](s)


# ---------------------------------------------------------------------------------------------- work
def work(case):
    layers, hq, hkv, dim, _ = SHAPES[case["shape"]]
    kind = case["kind"]
    if kind == "rotary":
        n = case["tokens"] * (hq + hkv)
        size = torch.finfo(TYPES[case["type"]]).bits // 8
        return {"bytes": 2 * n * dim * size + 4 * case["tokens"], "flops": 3 * n * case["rot"]}
    if kind == "append":
        rows = sum(chunk_lengths(case))
        tables = sum(pages_for(k) - (k - m) // PAGE for k, m in zip(keys_of(case), chunk_lengths(case)))
        return {"bytes": 2 * rows * (hq + 2 * hkv) * dim * 2 + 4 * tables, "flops": 3 * rows * (hq + hkv) * case["rot"]}
    if kind == "attention":
        pairs, read, rows, w = 0, 0, 0, case["window"]
        for m, n in zip(chunk_lengths(case), keys_of(case)):
            first = n - m  # position of the first new row
            seen = [min(p + 1, w) if w else p + 1 for p in range(first, n)]
            pairs += sum(seen)
            read += n - (max(0, first + 1 - w) if w else 0)
            rows += m
        return {"bytes": read * hkv * dim * 4 + 4 * read // PAGE + rows * hq * (dim * 4 + 4), "flops": 4 * pairs * hq * dim}
    tokens = table_tokens(case)
    entries = sum(pages_for(n) for n in tokens)
    total = entries + case["free"]
    if kind == "release":
        return {"bytes": 4 * entries + 8 * total, "flops": entries}
    slot = case["layers"] * 2 * hkv * dim * 2  # bytes of one token, all layers, K and V
    if kind == "fork":
        slots = sum(tokens) if case["deep"] else sum(n % PAGE for n in tokens)
    else:
        counts = [pages_for(n) for n in tokens]
        live = sum(counts) - sum(min(counts[i], counts[i - 1]) // 2 for i in range(1, len(counts), 2))
        slots = PAGE * live * (total - live) // total  # pages behind the front's share, tables permuted at random
    return {"bytes": 2 * slots * slot + 8 * entries + 8 * total, "flops": entries + total}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact_rotated(x, positions, case, inverse):
    """The rotation as a product of complex numbers, in 64 bits."""
    a = rope_args(case)
    rot, s = a["rot_dim"], a.get("factor", 1.0)
    f = []
    for i in range(rot // 2):
        theta = a["theta"] * (s ** (rot / (rot - 2.0)) if a["scaling"] == "base" else 1.0)
        w = math.exp(-2.0 * i / rot * math.log(theta))
        if a["scaling"] == "linear":
            w /= s
        if a["scaling"] == "bands":
            r = a["original"] * w / (2.0 * math.pi)
            ramp = min(1.0, max(0.0, (r - a["low"]) / (a["high"] - a["low"])))
            w = w * (ramp + (1.0 - ramp) / s)
        f.append(w)
    f = torch.tensor(f, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full((len(positions), rot // 2), a.get("magnitude", 1.0), dtype=torch.float64, device=DEV), positions.double()[:, None] * f)
    turn = turn.conj() if inverse else turn
    y = x.double().clone()
    first = slice(0, rot // 2) if a["layout"] == "half" else slice(0, rot, 2)
    second = slice(rot // 2, rot) if a["layout"] == "half" else slice(1, rot, 2)
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn[:, None]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact_attention(s):
    q, window = s["q"].double(), s["case"]["window"]
    hkv, dim = s["k_pages"].shape[1], s["k_pages"].shape[3]
    g, row = q.shape[1] // hkv, 0
    out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
    for m, n, table in zip(s["new"], s["keys"], s["tables"]):
        j, p = torch.arange(n, device=DEV), torch.arange(n - m, n, device=DEV)
        hidden = (j[None] > p[:, None]) | ((p[:, None] - j[None] >= window) if window else False)
        for h in range(hkv):
            k = s["k_pages"][table.long(), h].reshape(-1, dim)[:n].double()
            v = s["v_pages"][table.long(), h].reshape(-1, dim)[:n].double()
            for head in range(h * g, h * g + g):
                z = (q[row : row + m, head] @ k.T / math.sqrt(dim)).masked_fill_(hidden, -math.inf)
                l = torch.logsumexp(z, 1)
                out[row : row + m, head] = torch.exp(z - l[:, None]) @ v
                lse[row : row + m, head] = l
        row += m
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "rotary":
        return exact_rotated(s["q"], s["positions"], case, case["inverse"]), exact_rotated(s["k"], s["positions"], case, case["inverse"])
    if s["kind"] == "append":
        p = torch.cat([torch.arange(n - m, n, device=DEV) for m, n in zip(s["new"], s["keys"])])
        q, k = exact_rotated(s["q"], p, case, False), exact_rotated(s["k"], p, case, False)
        kp, vp, row = s["k_pages"].double(), s["v_pages"].double(), 0
        for m, n, table in zip(s["new"], s["keys"], s["tables"]):
            at = torch.arange(n - m, n, device=DEV)
            where = table.long()[at // PAGE]
            kp[where, :, at % PAGE] = k[row : row + m]
            vp[where, :, at % PAGE] = s["v"][row : row + m].double()
            row += m
        return q, kp, vp
    if s["kind"] == "attention":
        return exact_attention(s)
    return None  # whole numbers and copies: equal to the plain form's, nothing is computed in floating point
