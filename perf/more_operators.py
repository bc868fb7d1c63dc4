"""One decoding step's operators over a paged KV cache as cases for timing and comparison:
appending rotated keys and values, attention of the step's rows over the cache, and the
sampled commit of tokens.

The cache: pools of K and V [n_slots, H_kv * d_h] in blocks of `block` consecutive slots, and
a table of block ids for each request; position p of request b is slot
tables[b, p / block] * block + p % block.  With `own` false, run() computes an operator with
elementary torch operations; with `own` true it makes the package's calls.

Kinds
  append     rows of a fused projection's output: queries and keys are rotated at the row's
             position (half-split pairs), keys and values go to the position's slot; a row
             of position -1 is padding and is stored nowhere
  attention  `rows` queries of each request over the first key_len[row] positions of the
             request (all of them, or, `causal`, up to the row's own); a row with none gives
             zeros
  sample     for each row of logits: tokens ordered by logit (equal ones by index), weights
             exp((x - max) / temperature), the first top_k, of these the shortest run that
             holds top_p of their mass, of these the ones of at least min_p times the
             largest weight; the first token whose cumulative weight exceeds u times the
             kept mass is drawn and written to the token ids

Shapes are those of the package's workloads: LLaDA-8B's block (32 query and KV heads of 128),
Dream-7B's (28 on 4), the fp32 layers' heads, and a vocabulary of 126464.
"""

import math

import torch

own = False

LLADA = dict(heads=32, kv_heads=32, head_dim=128, dtype="bf16")
DREAM = dict(heads=28, kv_heads=4, head_dim=128, dtype="bf16")
F32 = dict(heads=4, kv_heads=2, head_dim=32, dtype="f32")
# a normalised row times an N(0, 0.02^2) projection of 4096 inputs
SPREAD = 1.28


def listed():
    return [
        # the next token of one user: a row behind a context of 1536 positions
        dict(name="append-llada-b1-token", kind="append", **LLADA, base=10000.0, block=64, batch=1, rows=1, fewer=0, first=1536),
        # prompts of unequal length, padded to the longest, grouped heads, short blocks
        dict(name="append-dream-b4-prompts", kind="append", **DREAM, base=10000.0, block=16, batch=4, rows=1331, fewer=77, first=0),
        # a long document of one user, far into its context
        dict(name="append-llada-document", kind="append", **LLADA, base=10000.0, block=64, batch=1, rows=8192, fewer=0, first=100003),
        # one new token of one user
        dict(name="attn-llada-b1-token", kind="attention", **LLADA, block=64, batch=1, rows=1, keys=1537, shorter=0, empty=0, causal=True, lse=False),
        # one new token of eight users with long contexts, grouped heads, short blocks
        dict(name="attn-dream-b8-token", kind="attention", **DREAM, block=16, batch=8, rows=1, keys=30011, shorter=1003, empty=0, causal=True, lse=True),
        # one new token of a serving batch, a place in it unused
        dict(name="attn-llada-b32-token", kind="attention", **LLADA, block=64, batch=32, rows=1, keys=4352, shorter=37, empty=1, causal=True, lse=False),
        # a block of 32 positions of four users with grouped heads, every row over the whole context
        dict(name="attn-dream-b4-block", kind="attention", **DREAM, block=32, batch=4, rows=32, keys=5120, shorter=11, empty=0, causal=False, lse=False),
        # a block of 32 positions of eight users
        dict(name="attn-llada-b8-block", kind="attention", **LLADA, block=64, batch=8, rows=32, keys=2432, shorter=0, empty=0, causal=False, lse=False),
        # the fp32 layer's heads: a few tokens, odd lengths, a block that is no power of two
        dict(name="attn-f32-tokens", kind="attention", **F32, block=24, batch=3, rows=5, keys=403, shorter=131, empty=0, causal=True, lse=True),
        # one token of one user
        dict(name="sample-b1-token", kind="sample", dtype="bf16", rows=1, vocab=126464, temperature=0.7, top_k=50, top_p=0.9, min_p=0.0, mixed=False),
        # a block of 32 positions of 32 users, each request with settings of its own
        dict(name="sample-b32-blocks", kind="sample", dtype="bf16", rows=1024, vocab=126464, temperature=0.9, top_k=400, top_p=0.95, min_p=0.02, mixed=True),
        # logits kept in 32 bits, an odd vocabulary, no cut: every token may be drawn
        dict(name="sample-f32-rows", kind="sample", dtype="f32", rows=67, vocab=50021, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["append", "attention", "attention", "sample"])
    if kind == "sample":
        vocab = log(1000, 160000)
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=max(1, min(log(1, 1024), 1024 * 126464 // (2 * vocab))),
                    vocab=vocab, temperature=round(rng.uniform(0.3, 1.6), 3), top_k=rng.choice([0, 1, log(2, 1000), log(2, 1000)]),
                    top_p=rng.choice([1.0, round(rng.uniform(0.05, 0.999), 3)]), min_p=rng.choice([0.0, round(rng.uniform(0.001, 0.3), 4)]),
                    mixed=rng.random() < 0.5)
    shape = dict(rng.choice([LLADA, DREAM, dict(heads=8, kv_heads=1, head_dim=128, dtype="bf16"),
                             dict(heads=16, kv_heads=8, head_dim=128, dtype="bf16"), F32,
                             dict(heads=4, kv_heads=4, head_dim=64, dtype="f32")]))
    block = rng.choice([1, 16, 16, 24, 32, 64, 64, 128, 256])
    batch = rng.choice([1, 2, 3, 5, 8, 13])
    if kind == "append":
        rows = max(1, log(1, 8192) // batch)
        return dict(kind=kind, **shape, base=rng.choice([10000.0, 500000.0]), block=block, batch=batch, rows=rows,
                    fewer=rng.randrange(1 + rows // (2 * batch)), first=rng.choice([0, log(1, 130000)]))
    rows = rng.choice([1, 1, 1, log(2, 9), 32, log(10, 64)])
    keys = max(rows, log(1, 32768))
    # no more than the largest listed case's pools
    keys = max(rows, min(keys, 32 * 4352 * 32 * 128 // (2 * batch * shape["kv_heads"] * shape["head_dim"])))
    return dict(kind=kind, **shape, block=block, batch=batch, rows=rows, keys=keys, shorter=rng.randrange(1 + (keys - rows) // batch),
                empty=rng.choice([0, 0, 1]) if batch > 1 else 0, causal=rng.random() < 0.6, lse=rng.random() < 0.5)


# ---------------------------------------------------------------------------- the plain forms
def slots_of(s, at):
    """Slots of positions at [batch, n] of each request (at >= 0)."""
    blocks = torch.gather(s["tables"].long(), 1, at // s["block"])
    return blocks * s["block"] + at % s["block"]


def rotated(x, pos, base):
    """x [n, heads, d] turned at pos [n]: angles in 64 bits, products in 32."""
    d = x.shape[-1]
    theta = torch.exp(torch.arange(d // 2, device=x.device, dtype=torch.float64) * (-2.0 * math.log(base) / d))
    angle = pos.double()[:, None] * theta
    cs, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    lo, hi = x[..., :d // 2].float(), x[..., d // 2:].float()
    return torch.cat([lo * cs - hi * sn, hi * cs + lo * sn], -1).to(x.dtype)


def plain_append(s):
    B, R, H, G, d = s["batch"], s["rows"], s["heads"], s["kv_heads"], s["head_dim"]
    pos = s["pos"].long()
    q, k, v = s["qkv"].split([H * d, G * d, G * d], 1)
    there = pos >= 0
    at = slots_of(s, pos.clamp(min=0).view(B, R)).view(-1)[there]
    s["k_pool"][at] = rotated(k.unflatten(1, (G, d)), pos, s["base"]).flatten(1)[there]
    s["v_pool"][at] = v[there]
    return rotated(q.unflatten(1, (H, d)), pos, s["base"]).flatten(1) * there[:, None]


def plain_attention(s):
    B, R, H, G, d = s["batch"], s["rows"], s["heads"], s["kv_heads"], s["head_dim"]
    S = max(s["keys"], 1)
    key_len = s["key_len"].long().view(B, R)
    at = torch.arange(S, device=key_len.device)[None, :].expand(B, S)
    at = torch.minimum(at, (key_len.amax(1, keepdim=True) - 1).clamp(min=0))
    slots = slots_of(s, at).clamp(min=0)
    k, v = (s[n][slots].view(B, S, G, d).permute(0, 2, 1, 3).float() for n in ("k_pool", "v_pool"))
    q = s["q"].view(B, R, G, H // G, d).permute(0, 2, 3, 1, 4).float().reshape(B, G, H // G * R, d)
    logit = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    logit = logit.view(B, G, H // G, R, S)
    logit.masked_fill_(torch.arange(S, device=at.device) >= key_len[:, None, None, :, None], -math.inf)
    top = logit.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp_(logit.sub_(top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, G, H // G * R, S), v.contiguous()).view(B, G, H // G, R, d) / torch.where(total == 0, 1.0, total)
    out = {"out": o.permute(0, 3, 1, 2, 4).reshape(B * R, H * d).to(s["q"].dtype)}
    if s["lse"]:
        out["lse"] = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).reshape(B * R, H)
    return out


def plain_sample(s):
    out, conf, prob = [], [], []
    rank = torch.arange(s["vocab"], device=s["x"].device)
    for rows in torch.arange(s["rows"], device=s["x"].device).split(256):
        x, idx = torch.sort(s["x"][rows].float(), dim=1, descending=True, stable=True)
        x = x.double()
        x -= x[:, :1].clone()
        t, u, p, m = (s[n][rows].double()[:, None] for n in ("temperature", "u", "top_p", "min_p"))
        k = s["top_k"][rows].long()[:, None]
        greedy = t <= 0
        w = torch.exp(x / torch.where(greedy, 1.0, t))
        w = torch.where((k > 0) & (rank >= k), 0.0, w)
        c = torch.cumsum(w, 1)
        keep = ((c - w < p * c[:, -1:]) | (p >= 1)) & (w >= m) & ((k <= 0) | (rank < k))
        keep[:, 0] = True
        n = keep.sum(1, keepdim=True)
        z = torch.gather(c, 1, n - 1)
        at = torch.minimum((c <= u * z).sum(1, keepdim=True), n - 1)
        at = torch.where(greedy, 0, at)
        out.append(torch.gather(idx, 1, at).squeeze(1))
        prob.append(torch.where(greedy, 1.0, torch.gather(w, 1, at) / z).squeeze(1))
        e = torch.exp(x)
        conf.append((torch.gather(e, 1, at) / e.sum(1, keepdim=True)).squeeze(1))
    out = torch.cat(out).int()
    s["ids"][s["commit_pos"].long()] = out
    return {"out": out, "conf": torch.cat(conf).float(), "prob": torch.cat(prob).float(), "ids": s["ids"]}


# ---------------------------------------------------------------------------- the cases' data
def type_of(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def values(g, shape, case, device):
    return (SPREAD * torch.randn(*shape, generator=g, device=device)).to(type_of(case))


def a_table(g, case, first, last, device):
    """tables [batch, blocks] for positions first[b] .. last[b] - 1, in blocks of a pool in any
    order, a few of which are nobody's; an entry that holds none of them is -1."""
    block, B = case["block"], case["batch"]
    f, n = torch.tensor(first, device=device) // block, -(-torch.tensor(last, device=device) // block)
    at = torch.arange(max(1, int(n.max())), device=device)[None, :]
    used = (at >= f[:, None]) & (at < n[:, None])
    total = int(used.sum()) + 3
    tables = torch.full(used.shape, -1, dtype=torch.int32, device=device)
    tables[used] = torch.randperm(total, generator=g, device=device)[:total - 3].to(torch.int32)
    return tables, total * block


def prepare(case, seed):
    device = "cuda"
    g = torch.Generator(device=device).manual_seed(int(seed))
    s = {k: v for k, v in case.items()}
    if case["kind"] == "sample":
        n, V = case["rows"], case["vocab"]
        x = 2.5 * torch.randn(n, V, generator=g, device=device)
        # the few tokens that fit the context stand out, in some rows more than in others
        ahead = torch.randint(V, (n, 24), generator=g, device=device)
        x.scatter_add_(1, ahead, 12 * torch.rand(n, 24, generator=g, device=device) * torch.rand(n, 1, generator=g, device=device))
        s["x"] = x.to(type_of(case))
        s["u"] = torch.rand(n, generator=g, device=device, dtype=torch.float64)
        f32 = dict(dtype=torch.float32, device=device)
        s["temperature"] = case["temperature"] * (0.75 + 0.5 * torch.rand(n, generator=g, device=device))
        s["top_k"] = torch.full((n,), case["top_k"], dtype=torch.int32, device=device)
        s["top_p"], s["min_p"] = torch.full((n,), case["top_p"], **f32), torch.full((n,), case["min_p"], **f32)
        if case["mixed"]:  # some rows draw without one cut or another, some take the largest
            which = torch.rand(4, n, generator=g, device=device)
            s["temperature"][which[0] < 0.1] = 0.0
            s["top_k"][which[1] < 0.3] = 0
            s["top_p"][which[2] < 0.3] = 1.0
            s["min_p"][which[3] < 0.5] = 0.0
        s["ids"] = torch.zeros(2 * n + 5, dtype=torch.int32, device=device)
        s["commit_pos"] = torch.randperm(2 * n + 5, generator=g, device=device)[:n].to(torch.int32)
        return s
    B, R, H, G, d = case["batch"], case["rows"], case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        rows = [R - b * case["fewer"] for b in range(B)]
        first = [case["first"] + 7 * b for b in range(B)]
        s["tables"], n_slots = a_table(g, case, first, [f + r for f, r in zip(first, rows)], device)
        at = torch.arange(R, device=device)[None, :]
        pos = torch.where(at < torch.tensor(rows, device=device)[:, None], at + torch.tensor(first, device=device)[:, None], -1)
        s["pos"] = pos.view(-1).to(torch.int32)
        s["qkv"] = values(g, (B * R, (H + 2 * G) * d), case, device)
    else:
        lens = [max(R, case["keys"] - b * case["shorter"]) if b < B - case["empty"] else 0 for b in range(B)]
        s["tables"], n_slots = a_table(g, case, [0] * B, lens, device)
        last = torch.tensor(lens, device=device)[:, None]
        ahead = R - 1 - torch.arange(R, device=device)[None, :] if case["causal"] else torch.zeros(1, R, dtype=torch.int64, device=device)
        s["key_len"] = (last - ahead).clamp(min=0).view(-1).to(torch.int32)
        s["q"] = values(g, (B * R, H * d), case, device)
    s["k_pool"], s["v_pool"] = values(g, (n_slots, G * d), case, device), values(g, (n_slots, G * d), case, device)
    if own:
        from paper_2608_26140_amd import acache as A

        s["dims"] = A.make_dims(H * d, H, G, d, 256, case["dtype"], rope_base=case.get("base", 10000.0))
        s["cache"] = A.PagedCache(s["k_pool"], s["v_pool"], case["block"], s["tables"])
        if case["kind"] == "attention":
            s["ws"] = A.paged_workspace(s["dims"], s["cache"], R)
    return s


# ---------------------------------------------------------------------------- a pass
def run(s):
    if not own:
        if s["kind"] == "sample":
            return plain_sample(s)
        if s["kind"] == "attention":
            return plain_attention(s)
        return {"q": plain_append(s), "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    from paper_2608_26140_amd import acache as A

    if s["kind"] == "sample":
        conf, prob = (torch.empty(s["rows"], dtype=torch.float32, device=s["x"].device) for _ in range(2))
        out = A.acache_sample_commit(s["x"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                     min_p=s["min_p"], conf=conf, prob=prob, commit_pos=s["commit_pos"], ids=s["ids"])
        return {"out": out, "conf": conf, "prob": prob, "ids": s["ids"]}
    H, G, d, R = s["heads"], s["kv_heads"], s["head_dim"], s["rows"]
    if s["kind"] == "append":
        q, k, v = s["qkv"].split([H * d, G * d, G * d], 1)
        q = A.acache_paged_append(s["dims"], s["cache"], k, v, s["pos"], R, q=q)
        return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    lse = torch.empty(s["q"].shape[0], H, device=s["q"].device) if s["lse"] else None
    out = A.acache_paged_attention(s["dims"], s["cache"], s["q"], s["key_len"], R, lse=lse, ws=s["ws"])
    return {"out": out, "lse": lse} if s["lse"] else {"out": out}


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "sample":
        return {"bytes": case["rows"] * (case["vocab"] * size + 4 * 8), "flops": 2 * case["rows"] * case["vocab"]}
    B, R, H, G, d = case["batch"], case["rows"], case["heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        rows = sum(R - b * case["fewer"] for b in range(B))
        blocks = -(-rows // case["block"])
        return {"bytes": 2 * rows * (H + 2 * G) * d * size + 4 * rows + 4 * blocks, "flops": 3 * rows * (H + G) * d}
    lens = [max(R, case["keys"] - b * case["shorter"]) for b in range(B - case["empty"])]
    pairs = sum(R * n - (R * (R - 1) // 2 if case["causal"] else 0) for n in lens)
    moved = 2 * sum(lens) * G * d * size + 4 * sum(-(-n // case["block"]) for n in lens) + 4 * B * R + 2 * B * R * H * d * size
    return {"bytes": moved + (4 * B * R * H if case["lse"] else 0), "flops": 4 * H * d * pairs}


# ---------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": exact_append, "attention": exact_attention, "sample": exact_sample}[case["kind"]](s)


def where(s, b, at):
    """Slots of request b's positions."""
    table = s["tables"][b].long()
    return table[torch.div(at, s["block"], rounding_mode="floor")] * s["block"] + torch.remainder(at, s["block"])


def exact_append(s):
    H, G, d, R = s["heads"], s["kv_heads"], s["head_dim"], s["rows"]
    j = torch.arange(d, device=s["qkv"].device)
    x = s["qkv"].double().view(-1, H + 2 * G, d)
    # an element's partner in its pair, and the sign with which it enters
    partner, sign = (j + d // 2) % d, torch.where(j < d // 2, -1.0, 1.0).double()
    freq = torch.pow(torch.tensor(s["base"], dtype=torch.float64, device=j.device), -(2.0 * (j % (d // 2))) / d)
    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    q = torch.zeros(x.shape[0], H, d, dtype=torch.float64, device=j.device)
    for b in range(s["batch"]):
        rows = torch.nonzero(s["pos"][b * R:(b + 1) * R] >= 0).squeeze(1) + b * R
        if rows.numel() == 0:
            continue
        pos = s["pos"][rows].long()
        angle = pos.double()[:, None, None] * freq
        turned = x[rows] * torch.cos(angle) + x[rows][..., partner] * sign * torch.sin(angle)
        q[rows] = turned[:, :H]
        slot = where(s, b, pos)
        k_pool[slot] = turned[:, H:H + G].flatten(1)
        v_pool[slot] = x[rows][:, H + G:].flatten(1)
    return {"q": q.flatten(1), "k_pool": k_pool, "v_pool": v_pool}


def exact_attention(s):
    H, G, d, R = s["heads"], s["kv_heads"], s["head_dim"], s["rows"]
    q = s["q"].double().view(-1, H, d)
    out = torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    lens = s["key_len"].tolist()
    for b in range(s["batch"]):
        top = max(lens[b * R:(b + 1) * R])
        if top == 0:
            continue
        slots = where(s, b, torch.arange(top, device=q.device))
        k, v = s["k_pool"][slots].view(top, G, d), s["v_pool"][slots].view(top, G, d)
        for n in set(lens[b * R:(b + 1) * R]) - {0}:
            rows = torch.tensor([r for r in range(b * R, (b + 1) * R) if lens[r] == n], device=q.device)
            for g in range(G):
                heads = slice(g * (H // G), (g + 1) * (H // G))
                logit = q[rows, heads].reshape(-1, d) @ k[:n, g].double().T / math.sqrt(d)
                lse[rows, heads] = torch.logsumexp(logit, 1).view(rows.numel(), -1)
                out[rows, heads] = (torch.softmax(logit, 1) @ v[:n, g].double()).view(rows.numel(), -1, d)
    res = {"out": out.flatten(1)}
    if s["lse"]:
        res["lse"] = lse
    return res


def exact_sample(s):
    out, conf, prob = [], [], []
    temperature, top_k, top_p, min_p, u = (s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    for r in range(s["rows"]):
        x = s["x"][r].double()
        soft = torch.softmax(x, 0)
        if temperature[r] <= 0:
            at, share = int(torch.nonzero(x == x.max())[0]), 1.0
        else:
            order = torch.argsort(-x, stable=True)
            w = torch.softmax(x / temperature[r], 0)[order]
            n = top_k[r] if 0 < top_k[r] < w.numel() else w.numel()
            mass = torch.cumsum(w[:n], 0)
            if top_p[r] < 1:
                n = min(n, 1 + int(torch.searchsorted(mass, top_p[r] * mass[-1])))
            n = max(1, min(n, int((w[:n] >= min_p[r] * w[0]).sum())))
            rank = min(int(torch.searchsorted(mass[:n], u[r] * mass[n - 1], right=True)), n - 1)
            at, share = int(order[rank]), w[rank] / mass[n - 1]
        out.append(at)
        conf.append(soft[at])
        prob.append(torch.as_tensor(share, dtype=torch.float64, device=x.device))
    out = torch.tensor(out, dtype=torch.int32, device=s["x"].device)
    ids = s["ids"].clone()
    ids[s["commit_pos"].long()] = out
    return {"out": out, "conf": torch.stack(conf), "prob": torch.stack(prob), "ids": ids}
