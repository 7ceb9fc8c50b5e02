"""Workloads of the paged KV cache: appending rotated keys, attention of new tokens, attention over selected pages.

Each case is one call that a decode step or a prompt makes for one layer.  A layer's cache is a pool of pages, K
[n_pages][Hkv][page][Dk] and V [n_pages][Hkv][page][Dv], a page table [B][width] of page ids, and per page the
smallest and largest value of every key dimension (k_min, k_max), which the selection reads.

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
    return [
        # the new token of a single request: the call that every layer of a batch-1 decode step makes, launch bound
        dict(gqa, name="append_token", kind="append", dtype="bf16", page=64, T=1, B=1, lo=5000, hi=5000, rot=128,
             interleaved=False, summaries=True),
        # a full decode batch far into long contexts, keys in 8 bits; some of its pages are completed
        dict(gqa, name="append_batch_fp8", kind="append", dtype="fp8", page=32, T=64, B=64, lo=100, hi=131071, rot=128,
             interleaved=False, summaries=True),
        # the prompts of three requests in one call, behind a long shared prefix
        dict(gqa, name="append_prompt", kind="append", dtype="bf16", page=64, T=8192, B=3, lo=60000, hi=100000, rot=128,
             interleaved=False, summaries=True),
        # prompts of no round length, keys wider than values, a part of each head rotated in neighbouring pairs
        dict(name="append_odd_fp32", kind="append", dtype="fp32", Hq=10, Hkv=10, Dk=192, Dv=128, page=16, T=777, B=5, lo=0,
             hi=900, rot=64, interleaved=True, summaries=False),
        # one request of a short conversation: latency
        dict(gqa, name="attend_token", kind="attend", dtype="bf16", page=64, B=1, lo=1000, hi=1000, window=0),
        # one request over a very long document: the whole card on one sequence
        dict(gqa, name="attend_long", kind="attend", dtype="bf16", page=64, B=1, lo=131072, hi=131072, window=0),
        # a serving batch of mixed lengths, an empty slot among them
        dict(gqa, name="attend_ragged", kind="attend", dtype="bf16", page=32, B=64, lo=1, hi=16384, window=0),
        # eight query heads a group, 8-bit cache, long contexts
        dict(name="attend_fp8", kind="attend", dtype="fp8", Hq=64, Hkv=8, Dk=128, Dv=128, page=64, B=32, lo=4096, hi=32768,
             window=0),
        # a small fp32 model with a sliding window
        dict(name="attend_window_fp32", kind="attend", dtype="fp32", Hq=20, Hkv=4, Dk=64, Dv=64, page=16, B=5, lo=300, hi=6000,
             window=1000),
        # a key and value head for each query head, keys wider than values
        dict(name="attend_wide_keys", kind="attend", dtype="bf16", Hq=10, Hkv=10, Dk=192, Dv=128, page=16, B=16, lo=1, hi=5001,
             window=0),
        # one long document, one page in thirty-two attended to
        dict(gqa, name="blocks_long", kind="blocks", dtype="bf16", page=64, B=1, lo=131072, hi=131072, n_sel=64, first=1, last=2),
        # a batch of long and short contexts, 8-bit cache: the short ones attend to all they have
        dict(name="blocks_batch_fp8", kind="blocks", dtype="fp8", Hq=64, Hkv=8, Dk=128, Dv=128, page=32, B=24, lo=900, hi=65536,
             n_sel=48, first=1, last=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "blocks", "blocks"])
    Hkv = rng.choice([1, 2, 4, 5, 8])
    group = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
    Dk, Dv = rng.choice([(64, 64), (80, 80), (96, 96), (128, 128), (128, 128), (128, 128), (192, 128), (256, 256)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp8", "fp8", "fp32"])
    page = rng.choice([16, 32, 64, 128])
    c = dict(kind=kind, dtype=dtype, Hq=Hkv * group, Hkv=Hkv, Dk=Dk, Dv=Dv, page=page)
    if kind == "append":
        if rng.random() < 0.5:
            B = _log_int(rng, 1, 200)
            c.update(T=B, B=B)
        else:
            c.update(T=_log_int(rng, 5, 4096), B=rng.choice([1, 2, 3, 5]))
        lo = _log_int(rng, 1, 60000)
        c.update(lo=lo, hi=_log_int(rng, lo, 120000), rot=rng.choice([Dk, Dk, Dk // 2]), interleaved=rng.random() < 0.4,
                 summaries=rng.random() < 0.6)
        return c
    B = _log_int(rng, 1, 96)
    budget = min(131072, 160 * 1024 * 1024 // (B * Hkv * (Dk + Dv)))  # tokens a sequence: below the largest listed case
    hi = max(2, _log_int(rng, min(600, budget), budget))
    c.update(B=B, lo=_log_int(rng, 1, hi), hi=hi)
    if kind == "attend":
        c.update(window=rng.choice([0, 0, 0, _log_int(rng, 1, hi)]))
    else:
        first, last = rng.choice([0, 1, 2]), rng.choice([1, 2, 4])
        c.update(n_sel=first + last + _log_int(rng, 1, 100), first=first, last=last)
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Lengths of a case's sequences (append: the position of each sequence's first new token): a matter of the case, not of the seed."""
    r = random.Random("%(lo)d %(hi)d %(B)d" % case)
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    if case["kind"] != "append" and case["B"] >= 8:
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


def _values(shape, dtype, g, std=1.0):
    """Normal values held in `dtype` (8 bits: codes, which a head's scale multiplies)."""
    if dtype != torch.float8_e4m3fn:
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype == torch.float32 else dtype) * std).to(dtype)
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) * (8.0 * std)).clamp(-FP8_MAX, FP8_MAX).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    io = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    B, Hq, Hkv, Dk, Dv, page = (case[n] for n in ("B", "Hq", "Hkv", "Dk", "Dv", "page"))
    s = dict(case)
    if case["kind"] == "append":
        seq, pos = _new_tokens(case)
        T = len(seq)
        width = max(pos) // page + 1
        held = sorted({(b, p // page) for b, p in zip(seq, pos)})
        n_pages = len(held) + 1
        order = torch.randperm(len(held), generator=g, device="cuda").to(torch.int32)
        table = torch.full((B, width), n_pages - 1, dtype=torch.int32, device="cuda")  # the rest of a sequence lies in a page that nobody writes
        table[torch.tensor([b for b, _ in held], device="cuda"), torch.tensor([p for _, p in held], device="cuda")] = order
        s.update(q=_values((T, Hq, Dk), io, g), k=_values((T, Hkv, Dk), io, g), v=_values((T, Hkv, Dv), io, g))
        s.update(seq=None if T == B else torch.tensor(seq, dtype=torch.int32, device="cuda"), pos=torch.tensor(pos, dtype=torch.int32, device="cuda"))
        s.update(ends=torch.tensor([t for t, p in enumerate(pos) if p % page == page - 1], dtype=torch.int64, device="cuda"))
        i = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
        s.update(inv_freq=(10000.0 ** (-2.0 * i / case["rot"])).float(), q_out=torch.empty_like(s["q"]))
    else:
        lens = _lengths(case)
        per = [-(-n // page) for n in lens]
        width = max(max(per), 1)
        n_pages = sum(per) + 1
        order = torch.randperm(n_pages - 1, generator=g, device="cuda").to(torch.int32)
        table = torch.full((B, width), n_pages - 1, dtype=torch.int32, device="cuda")
        used = torch.arange(width, device="cuda") < torch.tensor(per, device="cuda")[:, None]
        table[used] = order
        s.update(q=_values((B, Hq, Dk), io, g, 2.0), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), longest=max(lens))
    s.update(table=table, scale=1.0 / math.sqrt(Dk))
    s.update(k_pages=_values((n_pages, Hkv, page, Dk), dt, g), v_pages=_values((n_pages, Hkv, page, Dv), dt, g))
    if case["dtype"] == "fp8":
        s.update(k_scale=0.125 * (0.75 + 0.5 * torch.rand(Hkv, generator=g, device="cuda")),
                 v_scale=0.125 * (0.75 + 0.5 * torch.rand(Hkv, generator=g, device="cuda")))
    if case["kind"] == "blocks" or case.get("summaries"):
        held = io  # 8-bit codes are held exactly in bf16
        s.update(k_min=s["k_pages"].to(held).amin(2), k_max=s["k_pages"].to(held).amax(2))
    return s


# ------------------------------------------------------------------------------------------------ the library's calls
_handles = {}


def _own(s):
    """The handle of this geometry, which a program keeps, and the layer's pages as the calls take them."""
    import paper_2401_14361_amd as m
    key = (s["Hq"], s["Hkv"], s["Dk"], s["Dv"], s["page"], s["dtype"])
    B, width = s["table"].shape
    h = _handles.get(key)
    if h is None or h.max_batch < B or h.max_pages < width:
        h = _handles[key] = m.Kv(*key, max_batch=max(B, 64), max_pages=max(width, 4096))
    if "pages" not in s:
        s["pages"] = m.KvPages(h, s["k_pages"], s["v_pages"], k_min=s.get("k_min"), k_max=s.get("k_max"),
                               k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
    return m, h, s["pages"]


def run(s):
    if not own:
        return {"append": _append, "attend": _attend, "blocks": _blocks}[s["kind"]](s)
    m, h, pages = _own(s)
    if s["kind"] == "append":
        q = m.kv_append(h, pages, s["table"], s["pos"], s["q"], s["k"], s["v"], s["inv_freq"], seq=s["seq"],
                        interleaved=s["interleaved"], q_out=s["q_out"])
        return _written(s, q)
    if s["kind"] == "attend":
        out, lse = m.kv_attend(h, pages, s["table"], s["lens"], s["q"], s["scale"], window=s["window"], want_lse=True)
        return {"out": out, "lse": lse}
    out, lse, blocks = m.kv_attend_blocks(h, pages, s["table"], s["lens"], s["q"], s["scale"], s["n_sel"], keep_first=s["first"],
                                          keep_last=s["last"], want_lse=True, want_blocks=True)
    return {"out": out, "lse": lse, "blocks": blocks}


def _written(s, q):
    r = {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if s["summaries"]:
        r.update(k_min=s["k_min"], k_max=s["k_max"])
    return r


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
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


def _append(s):
    pos, page = s["pos"].long(), s["page"]
    angle = pos.double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    s["q_out"].copy_(_rotate(s["q"], cos, sin, s["rot"], s["interleaved"]))
    seq = torch.arange(pos.numel(), device=pos.device) if s["seq"] is None else s["seq"].long()
    at, row = s["table"][seq, pos // page].long(), pos % page
    dt = s["k_pages"].dtype
    s["k_pages"][at, :, row] = _held(_rotate(s["k"], cos, sin, s["rot"], s["interleaved"]), dt, s.get("k_scale"))
    s["v_pages"][at, :, row] = _held(s["v"].float(), dt, s.get("v_scale"))
    if s["summaries"]:
        done = at[s["ends"]]
        keys = s["k_pages"][done].float()
        s["k_min"][done] = keys.amin(2).to(s["k_min"].dtype)
        s["k_max"][done] = keys.amax(2).to(s["k_max"].dtype)
    return _written(s, s["q_out"])


def _softmax_over(s, q, keys, values, keep):
    """q [B][Hkv][G][Dk], keys and values [B][Hkv][n][D], keep [B][1 or Hkv][n] -> out [B][Hq][Dv], lse [B][Hq]."""
    scale = torch.full((1, 1, 1, 1), s["scale"], device=q.device)
    if "k_scale" in s:
        scale = scale * s["k_scale"][None, :, None, None]
        values = values * s["v_scale"][None, :, None, None]
    z = torch.matmul(q, keys.transpose(2, 3).contiguous()) * scale
    z = z.masked_fill(~keep[:, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, values) / torch.where(total == 0, torch.ones_like(total), total)
    lse = torch.log(total) + torch.where(total == 0, torch.full_like(top, -math.inf), top)
    B, Hq = q.shape[0], s["Hq"]
    return {"out": out.reshape(B, Hq, -1).to(s["q"].dtype), "lse": lse.reshape(B, Hq)}


def _attend(s):
    B, Hkv, page, n = s["B"], s["Hkv"], s["page"], s["longest"]
    j = torch.arange(n, device="cuda")
    at = s["table"][:, j // page].long()                                       # [B][n]
    keys = s["k_pages"][at, :, j % page].float().transpose(1, 2)               # [B][Hkv][n][Dk]
    values = s["v_pages"][at, :, j % page].float().transpose(1, 2).contiguous()
    lens = s["lens"].long()[:, None]
    keep = j < lens
    if s["window"]:
        keep = keep & (j >= lens - s["window"])
    q = s["q"].float().reshape(B, Hkv, s["Hq"] // Hkv, -1)
    return _softmax_over(s, q, keys, values, keep[:, None])


def _blocks(s):
    B, Hkv, page, width = s["B"], s["Hkv"], s["page"], s["table"].shape[1]
    table, lens = s["table"].long(), s["lens"].long()[:, None, None]
    n_blocks = (lens + page - 1) // page
    q = s["q"].double().reshape(B, Hkv, s["Hq"] // Hkv, -1)
    lo = s["k_min"][table].double().permute(0, 2, 3, 1).contiguous()           # [B][Hkv][Dk][width]
    hi = s["k_max"][table].double().permute(0, 2, 3, 1).contiguous()
    score = (torch.matmul(q.clamp(min=0), hi) + torch.matmul(q.clamp(max=0), lo)).amax(2)
    i = torch.arange(width, device="cuda")
    score = score.masked_fill((i < s["first"]) | (i >= n_blocks - s["last"]), math.inf).masked_fill(i >= n_blocks, -math.inf)
    take = min(s["n_sel"], width)
    chosen = score.sort(dim=-1, descending=True, stable=True).indices[..., :take]
    chosen = torch.where(chosen < n_blocks, chosen, torch.full_like(chosen, width)).sort(-1).values  # pages past the end go last
    there = chosen < width
    block = torch.where(there, chosen, torch.zeros_like(chosen))
    at = table[torch.arange(B, device="cuda")[:, None, None], block]           # [B][Hkv][take]
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    keys, values = s["k_pages"][at, head].float().flatten(2, 3), s["v_pages"][at, head].float().flatten(2, 3)
    j = (block[..., None] * page + torch.arange(page, device="cuda")).flatten(2)
    keep = (j < lens) & there.repeat_interleave(page, -1)
    r = _softmax_over(s, s["q"].float().reshape(B, Hkv, s["Hq"] // Hkv, -1), keys, values, keep)
    r["blocks"] = torch.full((B, Hkv, s["n_sel"]), -1, dtype=torch.int32, device="cuda")
    r["blocks"][..., :take] = torch.where(there, chosen, torch.full_like(chosen, -1)).int()
    return r


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    eb, io = BYTES[case["dtype"]], 4 if case["dtype"] == "fp32" else 2
    Hq, Hkv, Dk, Dv, page = (case[n] for n in ("Hq", "Hkv", "Dk", "Dv", "page"))
    if case["kind"] == "append":
        _, pos = _new_tokens(case)
        T = len(pos)
        b = T * ((2 * Hq + Hkv) * Dk + Hkv * Dv) * io + T * Hkv * (Dk + Dv) * eb + T * 8
        if case["summaries"]:
            ends = sum(p % page == page - 1 for p in pos)
            inside = max(0, ends * page - T) if T != case["B"] else ends * (page - 1)  # rows that the call has not just written
            b += inside * Hkv * Dk * eb + ends * Hkv * Dk * 2 * io
        return {"bytes": b, "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    lens = _lengths(case)
    ends = case["B"] * Hq * (Dk * io + Dv * io + 4)
    if case["kind"] == "attend":
        n = sum(min(x, case["window"] or x) for x in lens)
        return {"bytes": n * Hkv * (Dk + Dv) * eb + ends + sum(-(-x // page) for x in lens) * 4, "flops": 2 * n * Hq * (Dk + Dv)}
    per = [-(-x // page) for x in lens]
    n = sum(x if p <= case["n_sel"] else (case["n_sel"] - 1) * page + (x - 1) % page + 1 for x, p in zip(lens, per))
    scored = sum(p for p in per if p > case["n_sel"])  # where all pages are taken there is nothing to choose
    return {"bytes": n * Hkv * (Dk + Dv) * eb + scored * Hkv * Dk * 2 * io + ends + sum(per) * 4 + case["B"] * Hkv * case["n_sel"] * 4,
            "flops": 2 * n * Hq * (Dk + Dv) + 2 * scored * Hq * Dk}


# ------------------------------------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, Dk, page = s["Hq"], s["Hkv"], s["Dk"], s["page"]
    if case["kind"] == "append":
        rot, half = s["rot"], s["rot"] // 2
        first = list(range(0, rot, 2)) if s["interleaved"] else list(range(half))
        second = [d + 1 for d in first] if s["interleaved"] else [d + half for d in first]
        turn = torch.exp(1j * (s["pos"].double()[:, None] * s["inv_freq"].double()))[:, None]

        def turned(x):
            y = x.double().clone()
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            return y

        k, v = turned(s["k"]), s["v"].double()
        if case["dtype"] == "fp8":
            k = (k / s["k_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
            v = (v / s["v_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        r = {"q": turned(s["q"]), "k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
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
    B, G = s["B"], Hq // Hkv
    out = torch.zeros(B, Hq, s["Dv"], dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    blocks = torch.full((B, Hkv, s.get("n_sel", 1)), -1, dtype=torch.int32, device="cuda")
    k_scale = s["k_scale"].double() if "k_scale" in s else torch.ones(Hkv, dtype=torch.float64, device="cuda")
    v_scale = s["v_scale"].double() if "v_scale" in s else torch.ones(Hkv, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        nb = -(-n // page)
        mine = s["table"][b, :nb].long()
        for h in range(Hkv):
            q = s["q"][b, h * G:(h + 1) * G].double()
            if case["kind"] == "attend":
                begin = max(0, n - s["window"]) if s["window"] else 0
                j = torch.arange(begin, n, device="cuda")
            else:
                chosen = torch.arange(nb, device="cuda")
                if nb > s["n_sel"]:
                    a, z = q[:, None] * s["k_min"][mine, h].double(), q[:, None] * s["k_max"][mine, h].double()
                    bound = torch.maximum(a, z).sum(-1).max(0).values
                    bound[:s["first"]] = math.inf
                    bound[nb - s["last"]:] = math.inf
                    cut = bound.sort(descending=True).values[s["n_sel"] - 1]
                    above, equal = (bound > cut).nonzero()[:, 0], (bound == cut).nonzero()[:, 0]
                    chosen = torch.cat([above, equal[:s["n_sel"] - above.numel()]]).sort().values
                blocks[b, h, :chosen.numel()] = chosen.int()
                j = (chosen[:, None] * page + torch.arange(page, device="cuda")).flatten()
                j = j[j < n]
            keys = s["k_pages"][mine[j // page], h, j % page].double() * k_scale[h]
            z = s["scale"] * (q @ keys.T)
            l = torch.logsumexp(z, -1)
            out[b, h * G:(h + 1) * G] = torch.exp(z - l[:, None]) @ (s["v_pages"][mine[j // page], h, j % page].double() * v_scale[h])
            lse[b, h * G:(h + 1) * G] = l
    r = {"out": out, "lse": lse}
    if case["kind"] == "blocks":
        r["blocks"] = blocks
    return r
