"""Workloads of a served KV cache: appending keys and queries that are normed for each head, attention of a batch that shares prefixes,
attention that adds up what every cached token was given, and eviction by those sums.

Each case is one call that a decode step, a prompt or a cache that has grown too long makes for one layer.  A layer's cache is a pool of pages, K
[n_pages][Hkv][page][Dk] and V [n_pages][Hkv][page][Dv], and a page table [B][width] of page ids.

`own` chooses between the plain forms (elementary torch operations) and the library's entry points.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "fp32": 4, "fp8": 1}
FP8_MAX = 448.0


def listed():
    gqa = dict(Hq=32, Hkv=8, Dk=128, Dv=128)
    wide = dict(Hq=64, Hkv=8, Dk=128, Dv=128)
    return [
        # the new token of a single request, in a model that norms its queries and keys: once a layer and step, launch bound
        dict(gqa, name="norm_token", kind="norm", dtype="bf16", page=64, T=1, B=1, lo=5000, hi=5000, gone=0, rot=128,
             interleaved=False, per_head=False, summaries=False),
        # a decode batch over 8-bit caches that have evicted tokens: a token's angle is not that of its place
        dict(gqa, name="norm_batch_fp8", kind="norm", dtype="fp8", page=32, T=64, B=64, lo=100, hi=8191, gone=100000, rot=128,
             interleaved=False, per_head=False, summaries=True),
        # the prompts of three requests in one call; a norm's weights for every head, a part of each head rotated in neighbouring pairs
        dict(gqa, name="norm_prompt", kind="norm", dtype="bf16", page=64, T=8192, B=3, lo=0, hi=5000, gone=0, rot=64,
             interleaved=True, per_head=True, summaries=False),
        # four continuations of one short prompt: latency
        dict(gqa, name="shared_few", kind="shared", dtype="bf16", page=64, B=4, groups=1, plo=1024, phi=1024, lo=1, hi=64),
        # a serving batch behind one long system prompt, each request with a conversation of its own
        dict(gqa, name="shared_batch", kind="shared", dtype="bf16", page=64, B=64, groups=1, plo=32768, phi=32768, lo=1, hi=1024),
        # three prompts of their own length that several requests share each, in an 8-bit cache; the prefixes end inside pages
        dict(wide, name="shared_groups_fp8", kind="shared", dtype="fp8", page=32, B=48, groups=3, plo=3000, phi=20000, lo=0, hi=3000),
        # one request of a short conversation: latency
        dict(gqa, name="weights_token", kind="weights", dtype="bf16", page=64, B=1, lo=1000, hi=1000, window=0),
        # a serving batch of mixed lengths, an empty slot among them
        dict(gqa, name="weights_ragged", kind="weights", dtype="bf16", page=32, B=64, lo=1, hi=16384, window=0),
        # two very long documents in an 8-bit cache
        dict(wide, name="weights_long_fp8", kind="weights", dtype="fp8", page=64, B=2, lo=100000, hi=131072, window=0),
        # one request that has outgrown a small budget by a page
        dict(gqa, name="evict_page", kind="evict", dtype="bf16", page=64, B=1, lo=1088, hi=1088, keep=1024, first=4, last=256),
        # a batch after its prompts, cut down to a budget; what is shorter is moved whole
        dict(gqa, name="evict_batch", kind="evict", dtype="bf16", page=32, B=64, lo=700, hi=12000, keep=2048, first=4, last=128),
        # a long document's cache in 8 bits, one token in eight is kept
        dict(gqa, name="evict_long_fp8", kind="evict", dtype="fp8", page=64, B=1, lo=131072, hi=131072, keep=16384, first=16, last=1000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "shared", "shared", "weights", "evict"])
    Hkv = rng.choice([1, 2, 4, 5, 8])
    group = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    Dk, Dv = rng.choice([(64, 64), (80, 80), (96, 96), (128, 128), (128, 128), (128, 128), (192, 128), (256, 256)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp8", "fp8", "fp32"])
    page = rng.choice([16, 32, 64, 128])
    c = dict(kind=kind, dtype=dtype, Hq=Hkv * group, Hkv=Hkv, Dk=Dk, Dv=Dv, page=page)
    if kind == "norm":
        if rng.random() < 0.5:
            B = _log_int(rng, 1, 200)
            c.update(T=B, B=B)
        else:
            c.update(T=_log_int(rng, 5, 4096), B=rng.choice([1, 2, 3, 5]))
        lo = _log_int(rng, 1, 60000)
        c.update(lo=lo, hi=_log_int(rng, lo, 120000), gone=rng.choice([0, _log_int(rng, 1, 120000)]), rot=rng.choice([Dk, Dk, Dk // 2]),
                 interleaved=rng.random() < 0.4, per_head=rng.random() < 0.4, summaries=rng.random() < 0.4)
        return c
    if kind == "shared":
        B = _log_int(rng, 2, 96)
        # of a sequence's tokens: a plain form reads them all for each sequence; less work than the largest listed cases
        phi = _log_int(rng, 64, max(65, min(32768, 40_000_000 // (B * Hkv * group), 200_000_000 // (B * Hkv * (Dk + Dv)))))
        hi = _log_int(rng, 1, max(2, min(2048, 24_000_000 // (B * Hkv * (Dk + Dv)))))
        c.update(B=B, groups=rng.choice([1, 1, rng.randint(1, min(B, 12))]), plo=_log_int(rng, 1, phi), phi=phi, lo=rng.randint(0, hi), hi=hi)
        return c
    B = _log_int(rng, 1, 96)
    budget = min(131072, 120 * 1024 * 1024 // (B * Hkv * (Dk + Dv)))  # tokens a sequence: below the largest listed case
    hi = max(2, _log_int(rng, min(600, budget), budget))
    c.update(B=B, lo=_log_int(rng, 1, hi), hi=hi)
    if kind == "weights":
        c.update(window=rng.choice([0, 0, 0, _log_int(rng, 1, hi)]))
    else:
        first, last = rng.choice([0, 4, 50]), _log_int(rng, 1, 300)
        c.update(keep=first + last + _log_int(rng, 1, max(2, hi // 2)), first=first, last=last)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Lengths of a case's sequences (norm: the place of each sequence's first new token): a matter of the case, not of the seed."""
    r = random.Random("%(lo)d %(hi)d %(B)d" % case)
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    if case["kind"] in ("weights", "evict") and case["B"] >= 8:
        n[r.randrange(case["B"])] = 0  # a slot of the batch that holds no request
    return n


def _new_tokens(case):
    """(seq, pos) of an append's tokens: one a sequence, or runs of several, one sequence behind the other."""
    at, T, B = _lengths(case), case["T"], case["B"]
    if T == B:
        return list(range(B)), at
    share = [T // B + (b < T % B) for b in range(B)]
    seq = [b for b in range(B) for _ in range(share[b])]
    return seq, [at[b] + i for b in range(B) for i in range(share[b])]


def _groups(case):
    """(starts, prefixes): group g is the sequences starts[g] to starts[g + 1], whose first prefixes[g] tokens are the same."""
    r = random.Random("%(plo)d %(phi)d %(B)d %(groups)d" % case)
    cuts = sorted(r.sample(range(1, case["B"]), case["groups"] - 1))
    return [0, *cuts, case["B"]], [r.randint(case["plo"], case["phi"]) for _ in range(case["groups"])]


def _values(shape, dtype, g, std=1.0):
    """Normal values held in `dtype` (8 bits: codes, which a head's scale multiplies)."""
    if dtype != torch.float8_e4m3fn:
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype == torch.float32 else dtype) * std).to(dtype)
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * (8.0 * std)).clamp(-FP8_MAX, FP8_MAX).to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(B, places, n_extra, g):
    """A table that gives each of `places`, (sequence, number of the page) pairs, a page of its own in random order, and the ids of n_extra more."""
    n = len(places)
    order = torch.randperm(n + n_extra, generator=g, device="cuda").to(torch.int32)
    width = max((p for _, p in places), default=0) + 1
    table = torch.full((B, width), n + n_extra, dtype=torch.int32, device="cuda")  # the rest of a sequence: one more page, which nobody uses
    if places:
        table[_ints([b for b, _ in places]).long(), _ints([p for _, p in places]).long()] = order[:n]
    return table, order[n:], n + n_extra + 1


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    io = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    B, Hq, Hkv, Dk, Dv, page = (case[n] for n in ("B", "Hq", "Hkv", "Dk", "Dv", "page"))
    s = dict(case)
    if case["kind"] == "norm":
        seq, pos = _new_tokens(case)
        T = len(seq)
        table, _, n_pages = _table(B, sorted({(b, p // page) for b, p in zip(seq, pos)}), 0, g)
        s.update(q=_values((T, Hq, Dk), io, g, 3.0), k=_values((T, Hkv, Dk), io, g, 3.0), v=_values((T, Hkv, Dv), io, g))
        s.update(seq=None if T == B else _ints(seq), pos=_ints(pos), turn=None)
        if case["gone"]:  # tokens that the sequence has lost
            gone = torch.randint(0, case["gone"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["turn"] = s["pos"] + gone[_ints(seq).long()]
        s.update(ends=torch.tensor([t for t, p in enumerate(pos) if p % page == page - 1], dtype=torch.int64, device="cuda"))
        for n, H in (("q_weight", Hq), ("k_weight", Hkv)):
            s[n] = 1.0 + 0.3 * torch.randn((H, Dk) if case["per_head"] else (Dk,), generator=g, device="cuda")
        i = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
        s.update(inv_freq=(10000.0 ** (-2.0 * i / case["rot"])).float(), q_out=torch.empty_like(s["q"]), eps=1e-6)
    elif case["kind"] == "shared":
        starts, prefix = _groups(case)
        mine = _lengths(case)
        of = [g_ for g_ in range(case["groups"]) for _ in range(starts[g_ + 1] - starts[g_])]
        lens = [prefix[of[b]] + mine[b] for b in range(B)]
        first = [starts[of[b]] for b in range(B)]
        # whole pages of the prefix belong to the group's first sequence, and stand in every table; what lies behind them is each sequence's own
        held = [(b, p) for b in range(B) for p in range(0 if b == first[b] else prefix[of[b]] // page, -(-lens[b] // page))]
        table, _, n_pages = _table(B, held, 0, g)
        whole = torch.arange(table.shape[1], device="cuda") < _ints([prefix[of[b]] // page for b in range(B)])[:, None]
        table = torch.where(whole, table[_ints(first).long()], table).contiguous()
        s.update(starts=_ints(starts), prefix=_ints(prefix), lens=_ints(lens), longest=max(prefix), most=max(mine))
        most = max(starts[i + 1] - starts[i] for i in range(case["groups"]))
        s.update(members=_ints([[min(starts[i] + j, B - 1) for j in range(most)] for i in range(case["groups"])]).long(),
                 of=_ints(of).long(), at=_ints([b - first[b] for b in range(B)]).long())
        s.update(q=_values((B, Hq, Dk), io, g, 2.0))
    else:
        lens = _lengths(case)
        held = [(b, p) for b, n in enumerate(lens) for p in range(-(-n // page))]
        room = -(-case["keep"] // page) if case["kind"] == "evict" else 0
        table, spare, n_pages = _table(B, held, B * room, g)
        width = table.shape[1]
        s.update(lens=_ints(lens), longest=max(max(lens), 1))
        # what earlier steps have added up; many equal sums among the small ones
        w = torch.rand((B, Hkv, width * page), generator=g, device="cuda").pow(6.0)
        s["weights"] = torch.round(w * 8192.0) / 1024.0
        if case["kind"] == "weights":
            s.update(q=_values((B, Hq, Dk), io, g, 2.0))
        else:
            s.update(to_table=spare.reshape(B, room).contiguous(), to_weights=torch.rand((B, Hkv, room * page), generator=g, device="cuda"))
    s.update(table=table, scale=1.0 / math.sqrt(Dk))
    s.update(k_pages=_values((n_pages, Hkv, page, Dk), dt, g), v_pages=_values((n_pages, Hkv, page, Dv), dt, g))
    if case["dtype"] == "fp8":
        s.update(k_scale=0.125 * (0.75 + 0.5 * torch.rand(Hkv, generator=g, device="cuda")),
                 v_scale=0.125 * (0.75 + 0.5 * torch.rand(Hkv, generator=g, device="cuda")))
    if case.get("summaries"):
        s.update(k_min=s["k_pages"].to(io).amin(2), k_max=s["k_pages"].to(io).amax(2))  # 8-bit codes are held exactly in bf16
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
_handles = {}


def _own(s):
    """The handle of this geometry, which a program keeps, and the layer's pages as the calls take them."""
    import paper_2401_14361_amd as m
    key = (s["Hq"], s["Hkv"], s["Dk"], s["Dv"], s["page"], s["dtype"])
    B, width = s["table"].shape
    tokens = B * width * s["page"] if s["kind"] == "weights" else 0
    h = _handles.get(key)
    if h is None or h.max_batch < B or h.max_pages < width or h.max_weight_tokens < tokens:
        h = _handles[key] = m.Kv(*key, max_batch=max(B, 64), max_pages=max(width, 4096), max_sel=0, shared=True,
                                 max_weight_tokens=max(tokens, h.max_weight_tokens if h else 0))
    if "pages" not in s:
        s["pages"] = m.KvPages(h, s["k_pages"], s["v_pages"], k_min=s.get("k_min"), k_max=s.get("k_max"),
                               k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
    return m, h, s["pages"]


def run(s):
    if not own:
        return {"norm": _norm, "shared": _shared, "weights": _weights, "evict": _evict}[s["kind"]](s)
    m, h, pages = _own(s)
    if s["kind"] == "norm":
        q = m.kv_append_norm(h, pages, s["table"], s["pos"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["inv_freq"], eps=s["eps"],
                             seq=s["seq"], turn=s["turn"], interleaved=s["interleaved"], q_out=s["q_out"])
        return _written(s, q)
    if s["kind"] == "shared":
        out, lse = m.kv_attend_shared(h, pages, s["table"], s["lens"], s["starts"], s["prefix"], s["q"], s["scale"], want_lse=True)
        return {"out": out, "lse": lse}
    if s["kind"] == "weights":
        out, lse = m.kv_attend_weights(h, pages, s["table"], s["lens"], s["q"], s["scale"], s["weights"], window=s["window"], want_lse=True)
        return {"out": out, "lse": lse, "weights": s["weights"]}
    lens, kept = m.kv_evict(h, pages, s["table"], s["lens"], s["weights"], s["keep"], s["to_table"], s["to_weights"], keep_first=s["first"],
                            keep_last=s["last"])
    return _evicted(s, lens, kept)


def _written(s, q):
    r = {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if s["summaries"]:
        r.update(k_min=s["k_min"], k_max=s["k_max"])
    return r


def _evicted(s, lens, kept):
    return {"lens": lens, "kept": kept, "weights": s["to_weights"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, cos, sin, rot, interleaved):
    a, rest = x[..., :rot], x[..., rot:]
    c, s = cos[:, None], sin[:, None]
    if interleaved:
        x1, x2 = a[..., 0::2], a[..., 1::2]
        return torch.cat([torch.stack([x1 * c - x2 * s, x2 * c + x1 * s], -1).flatten(-2), rest], -1)
    x1, x2 = a[..., :rot // 2], a[..., rot // 2:]
    return torch.cat([x1 * c - x2 * s, x2 * c + x1 * s, rest], -1)


def _held(x, dtype, scale):
    if dtype != torch.float8_e4m3fn:
        return x.to(dtype)
    return (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX).to(dtype)


def _normed(x, weight, eps):
    x = x.float()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight


def _norm(s):
    pos, page = s["pos"].long(), s["page"]
    angle = (pos if s["turn"] is None else s["turn"]).double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    s["q_out"].copy_(_rotate(_normed(s["q"], s["q_weight"], s["eps"]), cos, sin, s["rot"], s["interleaved"]))
    seq = torch.arange(pos.numel(), device=pos.device) if s["seq"] is None else s["seq"].long()
    at, row = s["table"][seq, pos // page].long(), pos % page
    dt = s["k_pages"].dtype
    s["k_pages"][at, :, row] = _held(_rotate(_normed(s["k"], s["k_weight"], s["eps"]), cos, sin, s["rot"], s["interleaved"]), dt, s.get("k_scale"))
    s["v_pages"][at, :, row] = _held(s["v"].float(), dt, s.get("v_scale"))
    if s["summaries"]:
        done = at[s["ends"]]
        keys = s["k_pages"][done].float()
        s["k_min"][done] = keys.amin(2).to(s["k_min"].dtype)
        s["k_max"][done] = keys.amax(2).to(s["k_max"].dtype)
    return _written(s, s["q_out"])


def _gathered(s, table, begin, n):
    """Keys and values [rows of table][Hkv][n][D] of tokens begin (a number for each row) + 0 .. n - 1, in fp32."""
    j = begin[:, None] + torch.arange(n, device="cuda")
    at = torch.gather(table.long(), 1, (j // s["page"]).clamp(max=table.shape[1] - 1))
    keys = s["k_pages"][at, :, j % s["page"]].float().transpose(1, 2)
    values = s["v_pages"][at, :, j % s["page"]].float().transpose(1, 2).contiguous()
    if "v_scale" in s:
        values = values * s["v_scale"][None, :, None, None]
    return keys, values


def _logits(s, q, keys, keep):
    """q [N][Hkv][rows][Dk], keys [N][Hkv][n][Dk], keep [N][1][rows or 1][n] -> scaled logits, -inf where not kept."""
    z = torch.matmul(q, keys.transpose(2, 3).contiguous())
    scale = s["k_scale"][None, :, None, None] * s["scale"] if "k_scale" in s else s["scale"]
    return (z * scale).masked_fill(~keep, -math.inf)


def _shifted(z, top):
    return torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))


def _shared(s):
    B, Hkv, groups = s["B"], s["Hkv"], s["groups"]
    G, most = s["Hq"] // Hkv, s["members"].shape[1]
    q = s["q"].float().reshape(B, Hkv, G, -1)
    lens, members = s["lens"].long(), s["members"]
    # the prefixes, each once for all of its group's queries
    keys, values = _gathered(s, s["table"][members[:, 0]], torch.zeros(groups, dtype=torch.int64, device="cuda"), s["longest"])
    qg = q[members].transpose(1, 2).reshape(groups, Hkv, most * G, -1)
    upto = torch.minimum(lens[members], s["prefix"].long()[:, None]).repeat_interleave(G, 1)
    z = _logits(s, qg, keys, torch.arange(s["longest"], device="cuda") < upto[:, None, :, None])
    top_p = z.amax(-1, keepdim=True)
    p = _shifted(z, top_p)

    def of_sequences(x):
        return x.reshape(groups, Hkv, most, G, -1)[s["of"], :, s["at"]]

    sum_p, out_p, top_p = of_sequences(p.sum(-1, keepdim=True)), of_sequences(torch.matmul(p, values)), of_sequences(top_p)
    # what each sequence has of its own
    begin = s["prefix"].long()[s["of"]]
    n = max(s["most"], 1)
    keys, values = _gathered(s, s["table"], begin, n)
    z = _logits(s, q, keys, (torch.arange(n, device="cuda") < (lens - begin)[:, None])[:, None, None])
    top = torch.maximum(top_p, z.amax(-1, keepdim=True))
    p, f = _shifted(z, top), _shifted(top_p, top)
    total = sum_p * f + p.sum(-1, keepdim=True)
    out = (out_p * f + torch.matmul(p, values)) / torch.where(total == 0, torch.ones_like(total), total)
    lse = torch.log(total) + torch.where(total == 0, torch.full_like(top, -math.inf), top)
    return {"out": out.reshape(B, s["Hq"], -1).to(s["q"].dtype), "lse": lse.reshape(B, s["Hq"])}


def _weights(s):
    B, Hkv, n = s["B"], s["Hkv"], s["longest"]
    j, lens = torch.arange(n, device="cuda"), s["lens"].long()[:, None]
    keep = j < lens
    if s["window"]:
        keep = keep & (j >= lens - s["window"])
    keys, values = _gathered(s, s["table"], torch.zeros(B, dtype=torch.int64, device="cuda"), n)
    z = _logits(s, s["q"].float().reshape(B, Hkv, s["Hq"] // Hkv, -1), keys, keep[:, None, None])
    top = z.amax(-1, keepdim=True)
    p = _shifted(z, top)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    s["weights"][:, :, :n] += p.sum(2)
    lse = torch.log(total) + torch.where(total == 0, torch.full_like(top, -math.inf), top)
    return {"out": torch.matmul(p, values).reshape(B, s["Hq"], -1).to(s["q"].dtype), "lse": lse.reshape(B, s["Hq"]), "weights": s["weights"]}


def _evict(s):
    B, Hkv, page, keep = s["B"], s["Hkv"], s["page"], s["keep"]
    table, to_table, lens = s["table"].long(), s["to_table"].long(), s["lens"].long()[:, None, None]
    n = max(table.shape[1] * page, to_table.shape[1] * page)
    j = torch.arange(n, device="cuda")
    w = torch.nn.functional.pad(s["weights"], (0, n - s["weights"].shape[2]))
    w = w.masked_fill((j < s["first"]) | (j >= lens - s["last"]), math.inf).masked_fill(j >= lens, -math.inf)
    chosen = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    chosen = torch.where(chosen < lens, chosen, torch.full_like(chosen, n)).sort(-1).values  # what lies behind the sequence goes last
    there = chosen < n
    kept = torch.where(there, chosen, torch.full_like(chosen, -1)).int()
    room = to_table.shape[1] * page
    there, token = torch.nn.functional.pad(there, (0, room - keep)), torch.nn.functional.pad(chosen.masked_fill(~there, 0), (0, room - keep))
    s["to_weights"].copy_(torch.where(there, torch.gather(s["weights"], 2, token), s["to_weights"]))
    at = torch.gather(table, 1, (token // page).flatten(1)).reshape(token.shape)
    head = torch.arange(Hkv, device="cuda")[None, :, None]

    def moved(pages):
        """The rows that are kept, in their places; the other rows of those pages as they are."""
        D = pages.shape[-1]
        new = pages[at, head, token % page].reshape(B, Hkv, -1, page, D).transpose(1, 2)
        old = pages[to_table]
        if pages.dtype == torch.float8_e4m3fn:  # codes, bit for bit
            new, old = new.view(torch.uint8), old.view(torch.uint8)
        new = torch.where(there.reshape(B, Hkv, -1, page, 1).transpose(1, 2), new, old)
        pages[to_table] = new.contiguous().view(pages.dtype) if pages.dtype == torch.float8_e4m3fn else new

    moved(s["k_pages"])
    moved(s["v_pages"])
    return _evicted(s, s["lens"].clamp(max=keep), kept)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    eb, io = BYTES[case["dtype"]], 4 if case["dtype"] == "fp32" else 2
    B, Hq, Hkv, Dk, Dv, page = (case[n] for n in ("B", "Hq", "Hkv", "Dk", "Dv", "page"))
    if case["kind"] == "norm":
        _, pos = _new_tokens(case)
        T = len(pos)
        b = T * ((2 * Hq + Hkv) * Dk + Hkv * Dv) * io + T * Hkv * (Dk + Dv) * eb + T * (12 if case["gone"] else 8) + case["rot"] * 2
        b += (Hq + Hkv if case["per_head"] else 2) * Dk * 4
        if case["summaries"]:
            ends = sum(p % page == page - 1 for p in pos)
            inside = max(0, ends * page - T) if T != case["B"] else ends * (page - 1)  # rows that the call has not just written
            b += inside * Hkv * Dk * eb + ends * Hkv * Dk * 2 * io
        return {"bytes": b, "flops": T * (Hq + Hkv) * (3 * case["rot"] + 4 * Dk)}
    lens = _lengths(case)
    ends = B * Hq * (Dk * io + Dv * io + 4)
    if case["kind"] == "shared":
        starts, prefix = _groups(case)
        once = sum(prefix) + sum(lens)
        pages = sum(-(-p // page) for p in prefix) + sum(-(-x // page) for x in lens)
        each = sum(p * (starts[i + 1] - starts[i]) for i, p in enumerate(prefix)) + sum(lens)
        return {"bytes": once * Hkv * (Dk + Dv) * eb + ends + pages * 4, "flops": 2 * each * Hq * (Dk + Dv)}
    pages = sum(-(-x // page) for x in lens) * 4
    if case["kind"] == "weights":
        n = sum(min(x, case["window"] or x) for x in lens)
        return {"bytes": n * Hkv * ((Dk + Dv) * eb + 8) + ends + pages, "flops": 2 * n * Hq * (Dk + Dv)}
    kept = sum(min(x, case["keep"]) for x in lens)
    return {"bytes": sum(lens) * Hkv * 4 + kept * Hkv * (2 * (Dk + Dv) * eb + 4 + 4) + pages + B * -(-case["keep"] // page) * 4, "flops": sum(lens) * Hkv}


# ------------------------------------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    B, Hq, Hkv, Dk, Dv, page = (s[n] for n in ("B", "Hq", "Hkv", "Dk", "Dv", "page"))
    G = Hq // Hkv
    if case["kind"] == "norm":
        rot, half = s["rot"], s["rot"] // 2
        first = list(range(0, rot, 2)) if s["interleaved"] else list(range(half))
        second = [d + 1 for d in first] if s["interleaved"] else [d + half for d in first]
        angle = (s["pos"] if s["turn"] is None else s["turn"]).double()[:, None] * s["inv_freq"].double()
        turn = torch.exp(1j * angle)[:, None]

        def made(x, weight):
            y = x.double()
            y = weight.double() * y * ((y ** 2).sum(-1, keepdim=True) / Dk + s["eps"]) ** -0.5
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            return y

        k, v = made(s["k"], s["k_weight"]), s["v"].double()
        if case["dtype"] == "fp8":
            k = (k / s["k_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
            v = (v / s["v_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        r = {"q": made(s["q"], s["q_weight"]), "k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
        seq, pos = _new_tokens(case)
        at = s["table"].cpu()[seq, [p // page for p in pos]].cuda().long()
        row = torch.tensor([p % page for p in pos], device="cuda")
        for h in range(Hkv):
            r["k_pages"][at, h, row] = k[:, h]
            r["v_pages"][at, h, row] = v[:, h]
        if s["summaries"]:
            r.update(k_min=s["k_min"].double(), k_max=s["k_max"].double())
            for t in s["ends"].tolist():
                r["k_min"][at[t]] = r["k_pages"][at[t]].min(1).values
                r["k_max"][at[t]] = r["k_pages"][at[t]].max(1).values
        return r
    if case["kind"] == "evict":
        kept = torch.full((B, Hkv, s["keep"]), -1, dtype=torch.int32, device="cuda")
        weights, k, v = s["to_weights"].double(), s["k_pages"].double(), s["v_pages"].double()
        lens = []
        for b, n in enumerate(_lengths(case)):
            m = min(n, s["keep"])
            lens.append(m)
            for h in range(Hkv):
                chosen = torch.arange(n, device="cuda")
                if n > s["keep"]:
                    w = s["weights"][b, h, s["first"]:n - s["last"]]
                    free = s["keep"] - s["first"] - s["last"]
                    cut = w.sort(descending=True).values[free - 1] if free else math.inf
                    above, equal = (w > cut).nonzero()[:, 0], (w == cut).nonzero()[:, 0]
                    inner = torch.cat([above, equal[:free - above.numel()]]) + s["first"]
                    chosen = torch.cat([chosen[:s["first"]], inner.sort().values, chosen[n - s["last"]:]])
                if m == 0:
                    continue
                kept[b, h, :m] = chosen.int()
                weights[b, h, :m] = s["weights"][b, h, chosen].double()
                i = torch.arange(m, device="cuda")
                old, new = s["table"][b, chosen // page].long(), s["to_table"][b, i // page].long()
                k[new, h, i % page] = s["k_pages"][old, h, chosen % page].double()
                v[new, h, i % page] = s["v_pages"][old, h, chosen % page].double()
        return {"lens": _ints(lens), "kept": kept, "weights": weights, "k_pages": k, "v_pages": v}
    out = torch.zeros(B, Hq, Dv, dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    k_scale = s["k_scale"].double() if "k_scale" in s else torch.ones(Hkv, dtype=torch.float64, device="cuda")
    v_scale = s["v_scale"].double() if "v_scale" in s else torch.ones(Hkv, dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if case["kind"] == "weights" else None
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        begin = max(0, n - s["window"]) if s.get("window") else 0
        j = torch.arange(begin, n, device="cuda")
        at = s["table"][b, j // page].long()
        if case["kind"] == "shared":  # the prefix is what the group's first sequence holds
            group = int(s["of"][b])
            at = torch.where(j < s["prefix"][group], s["table"][int(s["starts"][group]), j // page].long(), at)
        for h in range(Hkv):
            keys = s["k_pages"][at, h, j % page].double() * k_scale[h]
            z = s["scale"] * (s["q"][b, h * G:(h + 1) * G].double() @ keys.T)
            l = torch.logsumexp(z, -1)
            p = torch.exp(z - l[:, None])
            out[b, h * G:(h + 1) * G] = p @ (s["v_pages"][at, h, j % page].double() * v_scale[h])
            lse[b, h * G:(h + 1) * G] = l
            if weights is not None:
                weights[b, h, begin:n] += p.sum(0)
    return {"out": out, "lse": lse} if weights is None else {"out": out, "lse": lse, "weights": weights}
