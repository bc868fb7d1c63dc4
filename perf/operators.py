"""The 8-bit KV cache's operators as cases for timing and comparison: storing rows into a
quantised cache, reading rows back, and attention over it.

The cache: codes [n_slots, H_kv * d_h] in e4m3 and, for every block of `block` consecutive
slots and KV head, one scale, a power of two (0: an empty block); an entry's value is code
times scale.  With `own` false, run() computes an operator with elementary torch operations
in 32 bits; with `own` true it makes the package's calls.

Kinds
  store      rows of K and V go to their slots: a block written whole, or still empty, takes
             the smallest scale that holds its new rows; one written in part keeps its scale
             unless the new rows need a larger one, and then the entries it keeps are rounded
             to that
  load       rows of slots back to the storage type
  attention  queries of a ragged batch against each request's view of the cache (a shared
             affix, the request's own slots in place of its anchors, its other positions)

Shapes are those of the package's workloads: LLaDA-8B's block (32 query and KV heads of
128), Dream-7B's (28 on 4) and the fp32 layers' heads.
"""

import math

import torch

own = False

LLADA = dict(heads=32, kv_heads=32, head_dim=128, dtype="bf16")
DREAM = dict(heads=28, kv_heads=4, head_dim=128, dtype="bf16")
F32 = dict(heads=4, kv_heads=2, head_dim=32, dtype="f32")
# a normalised row times an N(0, 0.02^2) projection of 4096 inputs
SPREAD = 1.28
MAX_CODE = 448.0
E_MIN, E_MAX = -117, 119


def listed():
    return [
        # a decode step of one request: its block of 32 positions overwrites the slots its refresh wrote
        dict(name="store-llada-block", kind="store", **LLADA, block=64, batch=1, rows=32, first=500, kept=717, slots=1792),
        # a refresh of four requests, grouped heads, private regions that begin and end inside a block
        dict(name="store-dream-refresh", kind="store", **DREAM, block=64, batch=4, rows=1843, first=37, kept=0, slots=11509),
        # the fp32 layer's rows, odd counts, a small block
        dict(name="store-f32-rows", kind="store", **F32, block=16, batch=2, rows=70, first=5, kept=90, slots=403),
        # the affix cache of a serving batch, materialised once
        dict(name="store-llada-affix", kind="store", **LLADA, block=64, batch=1, rows=8192, first=0, kept=0, slots=8192),
        # one request's private rows back (odd count, any order of blocks)
        dict(name="load-dream-rows", kind="load", **DREAM, block=64, batch=1, rows=1331, slots=6427),
        # the affix read back for a pass over its keys
        dict(name="load-llada-affix", kind="load", **LLADA, block=64, batch=1, rows=8192, slots=9000),
        # one user's decode step: 32 rows against 1024 affix and 512 own positions
        dict(name="attn-llada-b1-step", kind="attention", **LLADA, block=64, batch=1, rows=32, fewer=0, affix=1024,
             anchors=205, other=512, shorter=0, lse=False),
        # one row for each of eight requests, long contexts of their own, each of another length
        dict(name="attn-dream-b8-row", kind="attention", **DREAM, block=64, batch=8, rows=1, fewer=0, affix=0, anchors=0,
             other=30011, shorter=1003, lse=True),
        # a decode step of four requests with grouped heads and an affix of 4096
        dict(name="attn-dream-b4-step", kind="attention", **DREAM, block=64, batch=4, rows=32, fewer=0, affix=4096,
             anchors=819, other=1024, shorter=0, lse=False),
        # the serving batch's decode step: 32 requests of 32 rows share an affix of 8192
        dict(name="attn-llada-b32-step", kind="attention", **LLADA, block=64, batch=32, rows=32, fewer=0, affix=8192,
             anchors=1638, other=512, shorter=0, lse=False),
        # one user's refresh: anchors and own rows, 717 of them
        dict(name="attn-llada-b1-refresh", kind="attention", **LLADA, block=64, batch=1, rows=717, fewer=0, affix=1024,
             anchors=205, other=512, shorter=0, lse=True),
        # a refresh of eight requests, rows and keys of unequal number
        dict(name="attn-llada-b8-refresh", kind="attention", **LLADA, block=64, batch=8, rows=794, fewer=11, affix=2048,
             anchors=410, other=384, shorter=17, lse=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["store", "load", "attention", "attention"])
    block = rng.choice([16, 32, 64, 128, 256])
    bf16 = dict(rng.choice([LLADA, DREAM, dict(heads=8, kv_heads=1, head_dim=128, dtype="bf16"),
                            dict(heads=16, kv_heads=8, head_dim=128, dtype="bf16")]))
    if kind == "attention":
        batch = rng.choice([1, 2, 3, 5, 8, 13])
        affix = rng.choice([0, log(64, 8192)])
        anchors = int(affix * rng.choice([0.0, 0.1, 0.2, 0.4]))
        other = log(17, 2048)
        # no more work than the largest listed case (2 ** 37.9 products of a query and a key element)
        rows = max(1, min(log(1, 1024), int(6352 * 2432 * 32 / (batch * (affix + other) * bf16["heads"]))))
        return dict(kind=kind, **bf16, block=block, batch=batch, rows=rows, fewer=rng.randrange(1 + rows // (2 * batch)),
                    affix=affix, anchors=anchors, other=other, shorter=rng.randrange(1 + other // (2 * batch)),
                    lse=rng.random() < 0.5)
    shape = rng.choice([bf16, bf16, dict(F32), dict(heads=4, kv_heads=4, head_dim=64, dtype="f32")])
    batch = rng.choice([1, 2, 4, 7])
    rows = max(1, min(log(1, 8192) // batch, 8192 * 32 * 128 // (batch * shape["kv_heads"] * shape["head_dim"])))
    if kind == "load":
        return dict(kind=kind, **shape, block=block, batch=batch, rows=rows, slots=batch * rows + rng.randrange(1, 500))
    first = rng.randrange(300)
    kept = rng.choice([0, first + rows + rng.randrange(300)])
    return dict(kind=kind, **shape, block=block, batch=batch, rows=rows, first=first, kept=kept,
                slots=batch * (first + max(rows, kept - first)) + rng.randrange(500))


# ---------------------------------------------------------------------------- the plain forms
def power(e):
    """2^e of int32 exponents, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def exponent(amax):
    """The smallest e with amax <= 448 * 2^e, within the kept range (amax fp32, finite)."""
    return (((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 8 - 127).clamp(E_MIN, E_MAX)


def encode(x, e):
    return (x * power(-e)).clamp(-MAX_CODE, MAX_CODE).to(torch.float8_e4m3fn)


def plain_store(x, slots, codes, scales, block):
    """x [n, H, d] into codes [n_slots, H, d] (e4m3) and scales [n_blocks, H], in place."""
    n_slots, n_blocks = codes.shape[0], scales.shape[0]
    x, slots = x.float(), slots.long()
    at = slots // block
    amax = torch.zeros_like(scales).index_reduce_(0, at, x.abs().amax(-1), "amax")
    written = torch.zeros(n_blocks * block, dtype=torch.bool, device=x.device)
    written[n_slots:] = True  # past the last slot nothing is kept
    written[slots] = True
    count = torch.zeros(n_blocks, dtype=torch.int32, device=x.device).index_add_(0, at, torch.ones_like(at, dtype=torch.int32))
    touched = torch.nonzero(count).squeeze(1)
    old = scales[touched]
    fresh = written.view(n_blocks, block)[touched].all(1)[:, None] | (old == 0)
    need = exponent(amax[touched])
    was = (old.view(torch.int32) >> 23) - 127
    e = torch.where(fresh, need, torch.maximum(need, was))
    rest = touched[:, None] * block + torch.arange(block, device=x.device)  # the touched blocks' slots
    keep = ~written[rest]
    which, slot = torch.nonzero(keep, as_tuple=True)[0], rest[keep]
    left = codes[slot].float() * torch.where(old == 0, 0.0, power(was - e))[which][..., None]
    codes[slot] = left.clamp(-MAX_CODE, MAX_CODE).to(torch.float8_e4m3fn)
    all_e = torch.zeros_like(scales, dtype=torch.int32)
    all_e[touched] = e
    codes[slots] = encode(x, all_e[at][..., None])
    scales[touched] = power(e)


def plain_load(slots, codes, scales, block, dtype):
    slots = slots.long()
    return (codes[slots].float() * scales[slots // block][..., None]).to(dtype)


def plain_attention(s):
    """Requests side by side, padded to the longest: rows [B, R], keys [B, S]."""
    B, R, S = s["row_at"].shape[0], s["row_at"].shape[1], s["key_at"].shape[1]
    H, G, d = s["heads"], s["kv_heads"], s["head_dim"]
    slots = s["read_slots"].long()[s["key_at"]]  # [B, S]
    k, v = ((s[n + "_codes"][slots].float() * s[n + "_scales"][slots // s["block"]][..., None]).permute(0, 2, 1, 3)
            for n in ("k", "v"))  # [B, G, S, d]
    q = s["q"].view(-1, G, H // G, d)[s["row_at"]].float()  # [B, R, G, rep, d]
    q = q.permute(0, 2, 3, 1, 4).reshape(B, G, H // G * R, d)
    logit = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    logit.masked_fill_(~s["key_ok"][:, None, None, :], -math.inf)
    top = logit.amax(-1, keepdim=True)
    p = torch.exp_(logit.sub_(top))
    total = p.sum(-1, keepdim=True)
    o = (torch.matmul(p, v.contiguous()) / total).view(B, G, H // G, R, d).permute(0, 3, 1, 2, 4)
    out = {"out": o.reshape(B, R, H * d)[s["row_ok"]].to(s["q"].dtype)}
    if s["lse"]:
        out["lse"] = (top + torch.log(total)).view(B, G, H // G, R).permute(0, 3, 1, 2).reshape(B, R, H)[s["row_ok"]]
    return out


# ---------------------------------------------------------------------------- the cases' data
def type_of(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def values(g, case, n, device):
    """n rows of keys or values [n, H, d]: heads of unequal spread, as trained projections have."""
    H, d = case["kv_heads"], case["head_dim"]
    x = torch.randn(n, H, d, generator=g, device=device)
    x *= SPREAD * torch.exp(0.5 * torch.randn(H, 1, generator=g, device=device))
    return x.to(type_of(case))


def a_cache(g, case, n_slots, filled, device):
    """A cache whose first `filled` slots hold rows; the rest is empty."""
    blocks = -(-n_slots // case["block"])
    s = {}
    for n in ("k", "v"):
        codes = torch.zeros(n_slots, case["kv_heads"], case["head_dim"], dtype=torch.float8_e4m3fn, device=device)
        scales = torch.zeros(blocks, case["kv_heads"], device=device)
        if filled:
            plain_store(values(g, case, filled, device), torch.arange(filled, device=device), codes, scales, case["block"])
        s[n + "_codes"], s[n + "_scales"] = codes, scales
    return s


def prepare(case, seed):
    device = "cuda"
    g = torch.Generator(device=device).manual_seed(int(seed))
    s = {k: v for k, v in case.items()}
    B, rows = case["batch"], case["rows"]
    i32 = dict(dtype=torch.int32, device=device)
    if case["kind"] == "store":
        stride = (case["slots"] - case["first"]) // B
        s.update(a_cache(g, case, case["slots"], case["kept"], device))
        s["to"] = torch.cat([torch.arange(rows, **i32) + (case["first"] + b * stride) for b in range(B)])
        s["k"], s["v"] = values(g, case, B * rows, device), values(g, case, B * rows, device)
    elif case["kind"] == "load":
        s.update(a_cache(g, case, case["slots"], case["slots"], device))
        # runs of 16 slots in any order: what is private lies in pieces between what is shared
        runs = -(-case["slots"] // 16)
        order = torch.randperm(runs, generator=g, device=device)[:, None] * 16 + torch.arange(16, device=device)
        s["from"] = order.view(-1)[order.view(-1) < case["slots"]][:B * rows].to(torch.int32)
    else:
        L, k, other = case["affix"], case["anchors"], case["other"]
        per = k + other
        s.update(a_cache(g, case, L + B * per, L + B * per, device))
        # the view of acache_build_maps: request b's anchors and other positions have slots of their
        # own from L + b * per on, in ascending position, and the other affix positions are shared
        fresh = torch.ones(B, L + other, dtype=torch.bool, device=device)
        fresh[:, :L] = torch.rand(B, L, generator=g, device=device).argsort(1).argsort(1) < k
        own_slot = L + torch.arange(B, device=device)[:, None] * per + fresh.cumsum(1) - 1
        view = torch.where(fresh, own_slot, torch.arange(L + other, device=device)[None, :])
        n_rows = [rows - b * case["fewer"] for b in range(B)]
        n_keys = [L + other - b * case["shorter"] for b in range(B)]
        s["cu_rows"] = [sum(n_rows[:b]) for b in range(B + 1)]
        s["cu_keys"] = [sum(n_keys[:b]) for b in range(B + 1)]
        s["read_slots"] = torch.cat([view[b, :n_keys[b]] for b in range(B)]).to(torch.int32)
        s["q"] = (SPREAD * torch.randn(s["cu_rows"][B], case["heads"] * case["head_dim"], generator=g, device=device)).to(type_of(case))
        for what, cu, n in (("row", s["cu_rows"], n_rows), ("key", s["cu_keys"], n_keys)):
            at = torch.arange(n[0], device=device)[None, :].repeat(B, 1)
            ok = at < torch.tensor(n, device=device)[:, None]
            s[what + "_ok"], s[what + "_at"] = ok, torch.where(ok, at + torch.tensor(cu[:B], device=device)[:, None], 0)
    if own:
        from paper_2608_26140_amd import acache as A

        s["dims"] = A.make_dims(case["heads"] * case["head_dim"], case["heads"], case["kv_heads"], case["head_dim"], 256,
                                case["dtype"])
        flat = [s[n].view(torch.uint8).view(s[n].shape[0], -1) for n in ("k_codes", "v_codes")]
        s["pool"] = A.QuantPool(*flat, s["k_scales"], s["v_scales"], case["block"])
        n = s["q"].shape[0] if case["kind"] == "attention" else B * rows
        s["ws"] = A.quant_workspace(s["dims"], n, s["pool"])
    return s


# ---------------------------------------------------------------------------- a pass
def run(s):
    if s["kind"] == "store":
        if own:
            from paper_2608_26140_amd import acache as A

            A.acache_quant_store(s["dims"], s["pool"], s["k"].flatten(1), s["v"].flatten(1), s["to"], ws=s["ws"])
        else:
            plain_store(s["k"], s["to"], s["k_codes"], s["k_scales"], s["block"])
            plain_store(s["v"], s["to"], s["v_codes"], s["v_scales"], s["block"])
        return {n: s[n] for n in ("k_codes", "v_codes", "k_scales", "v_scales")}
    if s["kind"] == "load":
        if own:
            from paper_2608_26140_amd import acache as A

            k, v = A.acache_quant_load(s["dims"], s["pool"], s["from"])
            return {"k": k.view(s["from"].numel(), s["kv_heads"], s["head_dim"]), "v": v.view(s["from"].numel(), s["kv_heads"], s["head_dim"])}
        return {n: plain_load(s["from"], s[n + "_codes"], s[n + "_scales"], s["block"], type_of(s)) for n in ("k", "v")}
    if not own:
        return plain_attention(s)
    from paper_2608_26140_amd import acache as A

    lse = torch.empty(s["q"].shape[0], s["heads"], device=s["q"].device) if s["lse"] else None
    out = A.acache_quant_attention(s["dims"], s["cu_rows"], s["cu_keys"], s["q"], s["read_slots"], s["pool"], lse=lse, ws=s["ws"])
    return {"out": out, "lse": lse} if s["lse"] else {"out": out}


def work(case):
    B, H, G, d = case["batch"], case["heads"], case["kv_heads"], case["head_dim"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] != "attention":
        n = B * case["rows"]
        blocks = -(-n // case["block"])
        return {"bytes": 2 * n * G * d * (size + 1) + 4 * n + 2 * 4 * blocks * G, "flops": 0}
    rows = [case["rows"] - b * case["fewer"] for b in range(B)]
    keys = [case["affix"] + case["other"] - b * case["shorter"] for b in range(B)]
    # the shared slots once, each request's own once
    distinct = (case["affix"] if case["affix"] > case["anchors"] else 0)
    distinct += sum(case["anchors"] + case["other"] - b * case["shorter"] for b in range(B))
    moved = 2 * distinct * G * d + 2 * 4 * G * -(-distinct // case["block"]) + 4 * sum(keys) + 2 * sum(rows) * H * d * size
    return {"bytes": moved + (4 * sum(rows) * H if case["lse"] else 0),
            "flops": 4 * H * d * sum(r * n for r, n in zip(rows, keys))}


# ---------------------------------------------------------------------------- in 64 bits
def two_to(e):
    """2^e in float64 from its bits: pow and ldexp are not exact on every device."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def nearest(y):
    """The e4m3 value nearest to each y of float64, |y| <= 448, even significands at ties."""
    _, ex = torch.frexp(y)  # |y| in [2^(ex - 1), 2^ex)
    step = two_to((ex - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return exact_attention(s)
    out = {}
    for n in ("k", "v"):
        codes, scales = s[n + "_codes"].double(), s[n + "_scales"].double()
        if case["kind"] == "load":
            per_slot = scales.repeat_interleave(case["block"], 0)[:codes.shape[0]]
            out[n] = (codes * per_slot[..., None]).index_select(0, s["from"].long())
            continue
        row_of = torch.full((codes.shape[0],), -1, dtype=torch.int64, device=codes.device)
        row_of[s["to"].long()] = torch.arange(s["to"].numel(), device=codes.device)
        for b in range(scales.shape[0]):
            sl = slice(b * case["block"], min((b + 1) * case["block"], codes.shape[0]))
            new = row_of[sl] >= 0
            if not bool(new.any()):
                continue
            x = s[n][row_of[sl][new]].double()  # [rows, H, d]
            m, ex = torch.frexp(x.abs().amax((0, 2)))  # amax = 2 m * 2^(ex - 1)
            e = torch.where(2 * m <= 1.75, ex - 9, ex - 8).clamp(E_MIN, E_MAX)
            before, kept = scales[b].clone(), codes[sl][~new]
            if not bool(new.all()):
                e = torch.maximum(e, torch.where(before > 0, torch.frexp(before)[1] - 1, e))
            sc = two_to(e)
            part = codes[sl]
            part[~new] = nearest(kept * (before / sc)[:, None])
            part[new] = nearest((x / sc[:, None]).clamp(-MAX_CODE, MAX_CODE))
            codes[sl], scales[b] = part, sc
        out[n + "_codes"], out[n + "_scales"] = codes, scales
    return out


def exact_attention(s):
    H, G, d, block = s["heads"], s["kv_heads"], s["head_dim"], s["block"]
    q = s["q"].double().view(-1, H, d)
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    for b in range(s["batch"]):
        r0, r1 = s["cu_rows"][b], s["cu_rows"][b + 1]
        slots = s["read_slots"][s["cu_keys"][b]:s["cu_keys"][b + 1]].long()
        for g in range(G):
            k, v = (s[n + "_codes"][:, g][slots].double() * s[n + "_scales"][:, g][slots // block].double()[:, None]
                    for n in ("k", "v"))
            for h in range(g * (H // G), (g + 1) * (H // G)):
                logit = q[r0:r1, h] @ k.T / math.sqrt(d)
                lse[r0:r1, h] = torch.logsumexp(logit, 1)
                out[r0:r1, h] = torch.softmax(logit, 1) @ v
    res = {"out": out.view(-1, H * d)}
    if s["lse"]:
        res["lse"] = lse
    return res
