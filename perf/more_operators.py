"""More of the calls around a recovered cache, as cases to time and compare.

A service that continues recovered prefixes in 16-token pages, for decoders whose query and key heads are normed, whose local
layers keep the first tokens in sight, whose requests fork from one prefix, and whose answers are scored:

* ``norm``: RMS norms of query and key heads with the position rotation in the same pass (``Context.norm_rotary``), its
  gradient (``Context.norm_rotary_grad``), and the form that writes keys and values into the pages (``Context.cache_append``
  with gains).
* ``logprobs``: log probability of a given token, entropy and top alternatives of rows of logits (``Context.logprobs``), and
  the gradient with respect to the logits (``Context.logprobs_grad``).
* ``sinks``: attention of new rows over their requests' cached keys through a sliding window, the first few keys always in
  sight (``Context.chunk_attention`` with ``sinks``).
* ``prefix``: attention of requests that share a long prefix, whose keys and values are read once for all of them
  (``Context.prefix_attention``).

Head counts and vocabularies are those of the tiny decoder and of the two Qwen2.5 shapes, or drawn; page tables are random
permutations of the pool.
"""
import math

import torch

own = False

PAGE = 16
DEV = "cuda:0"
EPS = 1e-6

# query heads, kv heads, head dim, rope theta, vocabulary
SHAPES = {"tiny": (4, 2, 64, 1e4, 512), "1.5b": (12, 2, 128, 1e6, 151936), "7b": (28, 4, 128, 1e6, 152064)}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the next generated token of one conversation: latency
        dict(name="norm-row", kind="norm", shape="1.5b", tokens=1, rot=128, layout="half", type="bf16", top=16000),
        # a prompt of odd length, half of each head turned, pairs side by side
        dict(name="norm-odd", kind="norm", shape="7b", tokens=5003, rot=64, layout="interleaved", type="fp16", top=131072),
        # a training step's long sequence: gradients of heads and of the two gains
        dict(name="norm-16k-gradient", kind="norm-gradient", shape="7b", tokens=16384, rot=128, layout="half", type="bf16", top=16384),
        # two prompts' next turns and a few generated tokens, keys normed, turned and written into their pages
        dict(name="norm-append", kind="norm-append", shape="7b", chunks="1,2048,1,1501,1", keys_min=3001, keys_max=16384, rot=128, layout="half"),
        # one generated token and its alternatives: latency
        dict(name="logprobs-row", kind="logprobs", rows=1, vocab=152064, type="fp32", top=20, masked=False, padded=False),
        # a batch of sequences scored, padded rows without a token, a vocabulary part of which is ruled out
        dict(name="logprobs-rows", kind="logprobs", rows=2001, vocab=151936, type="bf16", top=8, masked=True, padded=True),
        # the policy gradient of a batch with an entropy term
        dict(name="logprobs-gradient", kind="logprobs-gradient", rows=1021, vocab=152064, type="fp32", padded=True),
        # a batch of generated tokens in a local layer
        dict(name="sinks-rows", kind="sinks", shape="7b", chunks="16x1", keys_min=4000, keys_max=16384, window=4096, sinks=4),
        # requests of every kind in one call, odd window and sinks
        dict(name="sinks-ragged", kind="sinks", shape="1.5b", chunks="5,1,517,1,130,64", keys_min=300, keys_max=8200, window=1001, sinks=131),
        # the next turn of a long conversation: matrix products
        dict(name="sinks-chunk", kind="sinks", shape="7b", chunks="4096", keys_min=16384, keys_max=16384, window=4096, sinks=16),
        # one token for each of many samples of one recovered prompt
        dict(name="prefix-rows", kind="prefix", shape="7b", groups="32x1", shared="15000", own_min=5, own_max=600),
        # drafted runs in two groups of samples, odd prefixes
        dict(name="prefix-drafts", kind="prefix", shape="1.5b", groups="7x5,5x3", shared="8003,3001", own_min=9, own_max=1500),
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


def groups_of(case):
    """(requests, new rows of each, shared keys) of each group."""
    return [(*map(int, g.split("x")), int(n)) for g, n in zip(case["groups"].split(","), case["shared"].split(","))]


def members_of(case):
    """(new rows, shared keys, keys) of each request, group by group: its own keys, the new rows' among them, follow the shared ones."""
    groups = groups_of(case)
    tails = spread_over(sum(g[0] for g in groups), case["own_min"], case["own_max"])
    flat = [(m, n) for count, m, n in groups for _ in range(count)]
    return [(m, n, n + max(t, m)) for (m, n), t in zip(flat, tails)]


def draw(rng):
    def spread(a, b):
        return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))

    kind = rng.choice(("norm", "norm-gradient", "norm-append", "logprobs", "logprobs", "logprobs-gradient", "sinks", "sinks", "prefix", "prefix"))
    shape = rng.choice(("tiny", "1.5b", "7b"))
    hq, hkv, d = SHAPES[shape][:3]
    rot, layout, kinds = rng.choice((d, d, d // 2, d // 4)), rng.choice(("half", "half", "interleaved")), ("bf16", "bf16", "fp16", "fp32")
    if kind in ("norm", "norm-gradient"):
        type = rng.choice(kinds)
        return dict(kind=kind, shape=shape, tokens=spread(1, 16384 if type != "fp32" else 8192), rot=rot, layout=layout, type=type, top=spread(200, 131072))
    if kind.startswith("logprobs"):
        vocab, type = rng.choice((spread(500, 152064), 512, 151936, 152064)), rng.choice(kinds)
        rows = spread(1, min(16384, 1021 * 152064 // vocab))
        c = dict(kind=kind, rows=rows, vocab=vocab, type=type, padded=rng.random() < 0.5)
        return dict(c, top=rng.choice((0, 1, 5, 20, 32)), masked=rng.random() < 0.3) if kind == "logprobs" else c
    if kind in ("norm-append", "sinks"):
        n = rng.choice((1, 1, 2, 3, 5, 8, 16, 32, 48))
        room, new = 3500, []  # new rows left
        for _ in range(n):
            m = rng.choice((1, 1, 1, spread(1, 16), spread(2, 3500)))
            new.append(max(1, min(m, room // 2 if len(new) else room)))
            room -= new[-1]
        if rng.random() < 0.3:
            new = [1] * n
        top = 16384 if n <= 4 else 16384 * 4 // n
        a, b = sorted((spread(16, top), spread(16, top)))
        c = dict(kind=kind, shape=shape, chunks=",".join(map(str, new)), keys_min=a, keys_max=b)
        return dict(c, rot=rot, layout=layout) if kind == "norm-append" else dict(c, window=spread(16, 4096), sinks=rng.choice((1, 4, spread(1, 256))))
    groups, shared = [], []
    for _ in range(rng.choice((1, 1, 2, 3))):
        groups.append("%dx%d" % (spread(2, 32), rng.choice((1, 1, 1, spread(1, 16)))))
        shared.append(str(spread(100, 15000 // (len(groups)))))
    a, b = sorted((spread(1, 600), spread(1, 600)))
    return dict(kind=kind, shape=shape, groups=",".join(groups), shared=",".join(shared), own_min=a, own_max=b)


# ---------------------------------------------------------------------------------------------- inputs
class Draws:
    """Seeded values on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=self.g)

    def uniform(self, shape):
        return torch.rand(shape, device=DEV, generator=self.g)

    def ints(self, n, top):
        return torch.randint(0, top, (n,), dtype=torch.int32, device=DEV, generator=self.g)

    def pages(self, n):
        return torch.randperm(n, device=DEV, generator=self.g).to(torch.int32)

    def gain(self, dim, dtype):
        return (1 + 0.1 * self.normal((dim,), torch.float32)).to(dtype)


def rope_args(case):
    return dict(head_dim=SHAPES[case["shape"]][2], rot_dim=case["rot"], theta=SHAPES[case["shape"]][3], layout=case["layout"])


def pages_for(n):
    return (n + PAGE - 1) // PAGE


def pool_of(d, s, total, hkv, dim):
    shape = (total, hkv, PAGE, dim)
    s["k_pages"] = d.normal(shape)
    # values share a mean a channel, as a trained layer's do
    s["v_pages"] = (d.normal(shape, torch.float32) + 0.5 * d.normal((hkv, 1, dim), torch.float32)).bfloat16()


def prepare(case, seed):
    d = Draws(seed)
    kind = case["kind"]
    s = {"case": case, "kind": kind}
    if kind.startswith("logprobs"):
        n, v, t = case["rows"], case["vocab"], TYPES[case["type"]]
        z = d.normal((n, v), t)
        # rows of every temper, from nearly flat to sharp
        z *= (0.5 + 4 * d.uniform((n, 1))).to(t)
        if case.get("masked"):
            z.masked_fill_(d.uniform((v,))[None] < 0.3, -math.inf)
        targets = d.ints(n, v)
        if case["padded"]:
            targets = torch.where(d.uniform((n,)) < 0.1, -1, targets)
        s.update(z=z, targets=targets.int(), logprob=torch.empty(n, device=DEV), entropy=torch.empty(n, device=DEV), lse=torch.empty(n, device=DEV))
        if kind == "logprobs":
            top = min(case["top"], v)
            s.update(ids=torch.empty(n, top, dtype=torch.int32, device=DEV), alternatives=torch.empty(n, top, device=DEV))
        else:
            # what the forward call left with the program, and what comes back from the loss
            e = torch.logsumexp(z.float(), 1)
            p = (z.float() - e[:, None]).exp_()
            s.update(lse=e, entropy=-(p.xlogy(p)).sum(1), g_logprob=d.normal((n,), torch.float32), g_entropy=0.01 * d.normal((n,), torch.float32), dz=torch.empty_like(z))
        return s
    hq, hkv, dim, _, _ = SHAPES[case["shape"]]
    if kind in ("norm", "norm-gradient"):
        # q and k as a fused projection leaves them: heads of one row side by side
        n, t = case["tokens"], TYPES[case["type"]]
        x = d.normal((n, hq + hkv, dim), t) * 2
        s.update(q=x[:, :hq], k=x[:, hq:], positions=d.ints(n, case["top"]), q_gain=d.gain(dim, t), k_gain=d.gain(dim, t))
        for a in ("q", "k"):
            s[a + "_out"] = torch.empty_like(s[a], memory_format=torch.contiguous_format)
            if kind == "norm-gradient":
                s[a + "_grad"] = d.normal(s[a].shape, t)
                s[a + "_dgain"] = torch.empty(dim, device=DEV)
        return s
    if kind == "prefix":
        members = members_of(case)
        groups = groups_of(case)
        fresh = [pages_for(k) - n // PAGE for _, n, k in members]  # a request's own pages: from the one that the prefix ends in
        whole = [n // PAGE for _, _, n in groups]
        perm = d.pages(sum(fresh) + sum(whole) + 5)
        own_pages, shared = perm[: sum(fresh)].split(fresh), perm[sum(fresh) : sum(fresh) + sum(whole)].split(whole)
        group = [g for g, (count, _, _) in enumerate(groups) for _ in range(count)]
        s.update(new=[m for m, _, _ in members], keys=[k for _, _, k in members], tables=[torch.cat((shared[g], p)) for g, p in zip(group, own_pages)])
        pool_of(d, s, len(perm), hkv, dim)
        # the slots that a fork copied: the same keys and values in every member's page
        first = {}
        for g, (m, n, k), t in zip(group, members, s["tables"]):
            lead = first.setdefault(g, t)
            if n % PAGE and lead is not t:
                for pages in (s["k_pages"], s["v_pages"]):
                    pages[t[n // PAGE].long(), :, : n % PAGE] = pages[lead[n // PAGE].long(), :, : n % PAGE]
    else:
        new, keys = chunk_lengths(case), keys_of(case)
        counts = [pages_for(k) for k in keys]
        perm = d.pages(sum(counts) + 5)
        s.update(new=new, keys=keys, tables=[t.contiguous() for t in perm[: sum(counts)].split(counts)])
        pool_of(d, s, len(perm), hkv, dim)
    rows = sum(s["new"])
    if kind == "norm-append":
        qkv = d.normal((rows, hq + 2 * hkv, dim)) * 2
        s.update(q=qkv[:, :hq], k=qkv[:, hq : hq + hkv], v=qkv[:, hq + hkv :], q_out=torch.empty(rows, hq, dim, dtype=torch.bfloat16, device=DEV))
        s.update(q_gain=d.gain(dim, torch.bfloat16), k_gain=d.gain(dim, torch.bfloat16))
    else:
        s.update(q=d.normal((rows, hq, dim)), out=torch.empty(rows, hq, dim, dtype=torch.bfloat16, device=DEV), lse=torch.empty(rows, hq, device=DEV))
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def turned(w, positions, a, inverse=False):
    """w [rows, heads, dim] in 32 bits, turned at ``positions``: angles in 64 bits."""
    rot = a["rot_dim"]
    f = a["theta"] ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    angle = positions.double()[:, None] * f[None]
    c, n = angle.cos().float()[:, None], (angle.sin() * (-1 if inverse else 1)).float()[:, None]
    if a["layout"] == "half":
        u, v, rest = w[..., : rot // 2], w[..., rot // 2 : rot], w[..., rot:]
        return torch.cat((u * c - v * n, v * c + u * n, rest), -1)
    u, v, rest = w[..., 0:rot:2], w[..., 1:rot:2], w[..., rot:]
    return torch.cat((torch.stack((u * c - v * n, v * c + u * n), -1).flatten(-2), rest), -1)


def normed(x, gain, positions, a):
    w = x.float()
    r = ((w * w).mean(-1, keepdim=True) + EPS).rsqrt()
    return turned(w * r * gain.float(), positions, a).to(x.dtype)


def plain_norm_gradient(s, name, a):
    x, u = s[name].float(), turned(s[name + "_grad"].float(), s["positions"], a, inverse=True)
    r = ((x * x).mean(-1, keepdim=True) + EPS).rsqrt()
    s[name + "_dgain"].copy_((u * x * r).sum((0, 1), dtype=torch.float64))
    v = u * s[name + "_gain"].float()
    s[name + "_out"].copy_(r * v - x * r**3 * (v * x).mean(-1, keepdim=True))
    return s[name + "_out"], s[name + "_dgain"]


def row_table(s):
    """Request and position of each new row, on the GPU."""
    new = torch.tensor(s["new"], device=DEV)
    pos0 = torch.tensor(s["keys"], device=DEV) - new
    b = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEV), new, output_size=sum(s["new"]))
    i = torch.arange(sum(s["new"]), device=DEV) - (new.cumsum(0) - new)[b]
    return b, pos0[b] + i, i


def padded_tables(s):
    return torch.nn.utils.rnn.pad_sequence(s["tables"], batch_first=True).long()


def plain_norm_append(s):
    a = rope_args(s["case"])
    b, p, _ = row_table(s)
    page, slot = padded_tables(s)[b, p // PAGE], p % PAGE
    s["q_out"].copy_(normed(s["q"], s["q_gain"], p, a))
    s["k_pages"][page, :, slot] = normed(s["k"], s["k_gain"], p, a)
    s["v_pages"][page, :, slot] = s["v"]
    return s["q_out"], s["k_pages"], s["v_pages"]


def plain_attention(s):
    """Every request padded to the longest: scores, row maxima, weights and their sums in 32 bits."""
    b, p, i = row_table(s)
    hq, dim = s["q"].shape[1:]
    hkv = s["k_pages"].shape[1]
    g, m, window, sinks = hq // hkv, max(s["new"]), s["case"].get("window", 0), s["case"].get("sinks", 0)
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
        seen &= (j > at[..., None] - window) | (j < sinks)
    z = (q @ k.transpose(-1, -2) * dim**-0.5).view(nb, hkv, g, m, n).masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    z = z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    o = (z.view(nb, hkv, g * m, n) @ v).view(nb, hkv, g, m, dim) / total
    lse = (top + total.log()).squeeze(-1)
    s["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(nb, m, hq, dim)[b, i])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(nb, m, hq)[b, i])
    return s["out"], s["lse"]


def plain_logprobs(s):
    z = s["z"].float()
    top = z.amax(1, keepdim=True)
    e = (z - top).exp_()
    total = e.sum(1)
    s["lse"].copy_(top[:, 0] + total.log())
    t = s["targets"].long()
    s["logprob"].copy_(torch.where(t < 0, 0.0, z.gather(1, t.clamp(min=0)[:, None])[:, 0] - s["lse"]))
    s["entropy"].copy_(total.log() - (e * torch.where(e > 0, z - top, 0.0)).sum(1) / total)
    n = s["ids"].shape[1]
    # equal values in order of their index: one whole number orders both
    bits = (z + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2**32 + (z.shape[1] - torch.arange(z.shape[1], device=DEV))
    s["ids"].copy_(order.topk(n, 1).indices)
    s["alternatives"].copy_(z.gather(1, s["ids"].long()) - s["lse"][:, None])
    return s["logprob"], s["entropy"], s["lse"], s["ids"], s["alternatives"]


def plain_logprobs_gradient(s):
    l = s["z"].float() - s["lse"][:, None]
    p = l.exp()
    t = s["targets"].long()
    g = torch.where(t < 0, 0.0, s["g_logprob"])
    d = -p * (g[:, None] + s["g_entropy"][:, None] * (l + s["entropy"][:, None]))
    d.scatter_add_(1, t.clamp(min=0)[:, None], g[:, None])
    s["dz"].copy_(d)
    return s["dz"]


# ---------------------------------------------------------------------------------------------- the framework's calls
HELD = {}


def held(s):
    """What a program keeps across its layers and steps: the context, the pool, a step's chunks, a workspace."""
    import paper_2609_30884_gb300 as crf

    if "ctx" not in HELD:
        HELD["ctx"] = crf.Context(0)
    ctx, case, kind = HELD["ctx"], s["case"], s["kind"]
    h = {"ctx": ctx}
    if kind.startswith("norm"):
        h["rope"] = crf.Rope(**rope_args(case))
    if kind == "norm-gradient":
        h["ws"] = ctx.norm_rotary_workspace(h["rope"], s["q"].shape[0])
    if kind in ("norm-append", "sinks", "prefix"):
        h["pool"] = crf.KVPool([s["k_pages"]], [s["v_pages"]])
        h["chunks"] = crf.Chunks(s["tables"], s["new"], [k - m for k, m in zip(s["keys"], s["new"])])
    if kind == "sinks":
        h["ws"] = ctx.chunk_attention_workspace(h["pool"], h["chunks"], s["q"].shape[1], window=case["window"], sinks=case["sinks"])
    if kind == "prefix":
        h["prefixes"] = crf.Prefixes([count for count, _, _ in groups_of(case)], [n for _, _, n in groups_of(case)])
        h["ws"] = ctx.prefix_attention_workspace(h["pool"], h["chunks"], h["prefixes"], s["q"].shape[1])
    return h


def own_run(s):
    if "held" not in s:
        s["held"] = held(s)
    h, kind = s["held"], s["kind"]
    ctx = h["ctx"]
    if kind == "norm":
        ctx.norm_rotary(h["rope"], s["positions"], s["q"], s["q_gain"], out=s["q_out"], k=s["k"], k_gain=s["k_gain"], k_out=s["k_out"], eps=EPS)
        return s["q_out"], s["k_out"]
    if kind == "norm-gradient":
        ctx.norm_rotary_grad(h["rope"], s["positions"], s["q"], s["q_gain"], s["q_grad"], s["q_out"], s["q_dgain"], h["ws"], k=s["k"], k_gain=s["k_gain"], k_grad=s["k_grad"], k_dx=s["k_out"], k_dgain=s["k_dgain"], eps=EPS)
        return s["q_out"], s["q_dgain"], s["k_out"], s["k_dgain"]
    if kind == "norm-append":
        ctx.cache_append(h["pool"], 0, h["chunks"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=h["rope"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)
        return s["q_out"], s["k_pages"], s["v_pages"]
    if kind == "logprobs":
        ctx.logprobs(s["z"], s["targets"], logprob=s["logprob"], entropy=s["entropy"], lse=s["lse"], top_ids=s["ids"], top_logprobs=s["alternatives"])
        return s["logprob"], s["entropy"], s["lse"], s["ids"], s["alternatives"]
    if kind == "logprobs-gradient":
        ctx.logprobs_grad(s["z"], s["targets"], s["lse"], s["dz"], g_logprob=s["g_logprob"], entropy=s["entropy"], g_entropy=s["g_entropy"])
        return s["dz"]
    if kind == "sinks":
        ctx.chunk_attention(h["pool"], 0, h["chunks"], s["q"], s["out"], h["ws"], lse=s["lse"], window=s["case"]["window"], sinks=s["case"]["sinks"])
        return s["out"], s["lse"]
    ctx.prefix_attention(h["pool"], 0, h["chunks"], h["prefixes"], s["q"], s["out"], h["ws"], lse=s["lse"])
    return s["out"], s["lse"]


def run(s):
    if own:
        return own_run(s)
    kind = s["kind"]
    if kind == "norm":
        a = rope_args(s["case"])
        s["q_out"].copy_(normed(s["q"], s["q_gain"], s["positions"], a))
        s["k_out"].copy_(normed(s["k"], s["k_gain"], s["positions"], a))
        return s["q_out"], s["k_out"]
    if kind == "norm-gradient":
        a = rope_args(s["case"])
        return (*plain_norm_gradient(s, "q", a), *plain_norm_gradient(s, "k", a))
    return {"norm-append": plain_norm_append, "logprobs": plain_logprobs, "logprobs-gradient": plain_logprobs_gradient, "sinks": plain_attention, "prefix": plain_attention}[kind](s)


# ---------------------------------------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind.startswith("logprobs"):
        n, v, size = case["rows"], case["vocab"], torch.finfo(TYPES[case["type"]]).bits // 8
        if kind == "logprobs":
            return {"bytes": n * v * size + n * (16 + 8 * min(case["top"], v)), "flops": 4 * n * v}
        return {"bytes": 2 * n * v * size + 20 * n, "flops": 5 * n * v}
    hq, hkv, dim, _, _ = SHAPES[case["shape"]]
    if kind in ("norm", "norm-gradient"):
        n = case["tokens"] * (hq + hkv)
        size = torch.finfo(TYPES[case["type"]]).bits // 8
        if kind == "norm":
            return {"bytes": 2 * n * dim * size + 4 * case["tokens"] + 2 * dim * size, "flops": n * (4 * dim + 3 * case["rot"])}
        return {"bytes": 3 * n * dim * size + 4 * case["tokens"] + 2 * dim * (size + 4), "flops": n * (9 * dim + 3 * case["rot"])}
    if kind == "norm-append":
        rows = sum(chunk_lengths(case))
        tables = sum(pages_for(k) - (k - m) // PAGE for k, m in zip(keys_of(case), chunk_lengths(case)))
        return {"bytes": 2 * rows * (hq + 2 * hkv) * dim * 2 + 4 * tables + 4 * dim, "flops": rows * (hq + hkv) * (4 * dim + 3 * case["rot"])}
    pairs, read, rows = 0, 0, 0
    if kind == "sinks":
        w, first = case["window"], case["sinks"]
        for m, n in zip(chunk_lengths(case), keys_of(case)):
            start = n - m  # position of the first new row
            pairs += sum(min(p + 1, w) + min(first, max(0, p + 1 - w)) for p in range(start, n))
            read += n - max(0, max(0, start + 1 - w) - first)
            rows += m
    else:
        for m, shared, n in members_of(case):
            pairs += sum(range(n - m + 1, n + 1))
            read += n - shared
            rows += m
        read += sum(n for _, _, n in groups_of(case))
    return {"bytes": read * hkv * dim * 4 + 4 * read // PAGE + rows * hq * (dim * 4 + 4), "flops": 4 * pairs * hq * dim}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact_normed(x, gain, positions, case):
    """x / rms(x) times the gain, its pairs turned as complex numbers, in 64 bits (x a leaf or not)."""
    a = rope_args(case)
    rot, dim = a["rot_dim"], a["head_dim"]
    f = torch.tensor([math.exp(-2.0 * i / rot * math.log(a["theta"])) for i in range(rot // 2)], dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones((len(positions), rot // 2), dtype=torch.float64, device=DEV), positions.double()[:, None] * f)[:, None]
    y = x * gain / torch.sqrt(x.square().sum(-1, keepdim=True) / dim + EPS)
    pairs = y[..., :rot]
    pairs = torch.stack((pairs[..., : rot // 2], pairs[..., rot // 2 :]), -1) if a["layout"] == "half" else pairs.unflatten(-1, (rot // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = torch.cat((z[..., 0], z[..., 1]), -1) if a["layout"] == "half" else z.flatten(-2)
    return torch.cat((z, y[..., rot:]), -1)


def exact_attention(s):
    q, window, sinks = s["q"].double(), s["case"].get("window", 0), s["case"].get("sinks", 0)
    hkv, dim = s["k_pages"].shape[1], s["k_pages"].shape[3]
    g, row = q.shape[1] // hkv, 0
    out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
    for m, n, table in zip(s["new"], s["keys"], s["tables"]):
        j, p = torch.arange(n, device=DEV), torch.arange(n - m, n, device=DEV)
        hidden = (j[None] > p[:, None]) | ((p[:, None] - j[None] >= window) & (j[None] >= sinks) if window else False)
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
    kind = s["kind"]
    if kind == "norm":
        return tuple(exact_normed(s[a].double(), s[a + "_gain"].double(), s["positions"], case) for a in ("q", "k"))
    if kind == "norm-gradient":
        got = []
        for a in ("q", "k"):
            x, gain = s[a].double().requires_grad_(), s[a + "_gain"].double().requires_grad_()
            got += torch.autograd.grad((exact_normed(x, gain, s["positions"], case) * s[a + "_grad"].double()).sum(), (x, gain))
        return tuple(got)
    if kind == "norm-append":
        p = torch.cat([torch.arange(n - m, n, device=DEV) for m, n in zip(s["new"], s["keys"])])
        q, k = exact_normed(s["q"].double(), s["q_gain"].double(), p, case), exact_normed(s["k"].double(), s["k_gain"].double(), p, case)
        kp, vp, row = s["k_pages"].double(), s["v_pages"].double(), 0
        for m, n, table in zip(s["new"], s["keys"], s["tables"]):
            at = torch.arange(n - m, n, device=DEV)
            where = table.long()[at // PAGE]
            kp[where, :, at % PAGE] = k[row : row + m]
            vp[where, :, at % PAGE] = s["v"][row : row + m].double()
            row += m
        return q, kp, vp
    if kind == "logprobs":
        z, parts = s["z"], []
        for i in range(0, len(z), 128):
            l = torch.log_softmax(z[i : i + 128].double(), 1)
            t = s["targets"][i : i + 128].long()
            lp = torch.where(t < 0, 0.0, l.gather(1, t.clamp(min=0)[:, None])[:, 0])
            p = l.exp()
            parts.append((lp, -torch.xlogy(p, p).sum(1), torch.logsumexp(z[i : i + 128].double(), 1), l.topk(s["ids"].shape[1], 1).values))
        lp, h, e, top = (torch.cat(x) for x in zip(*parts))
        return lp, h, e, None, top
    if kind == "logprobs-gradient":
        # of sum g_logprob logprob + g_entropy entropy, by differentiation
        got = torch.empty_like(s["z"], dtype=torch.float64)
        for i in range(0, len(got), 64):
            z = s["z"][i : i + 64].double().requires_grad_()
            l = torch.log_softmax(z, 1)
            t = s["targets"][i : i + 64].long()
            lp = torch.where(t < 0, 0.0, l.gather(1, t.clamp(min=0)[:, None])[:, 0])
            loss = (lp * s["g_logprob"][i : i + 64].double()).sum() - ((l.exp() * l).sum(1) * s["g_entropy"][i : i + 64].double()).sum()
            got[i : i + 64] = torch.autograd.grad(loss, z)[0]
        return got
    return exact_attention(s)
