"""Cases, inputs, plain forms and exact values for the operators between a prompt and its tokens: attention over whole prompts of
different lengths laid end to end, attention of a chunk of new tokens over a paged cache with a shared prefix, and the draw of
the next token (temperature, top-k, top-p, min-p, guidance) from given random numbers.

A pool is [n_pages][n_kv_heads][page_rows][row_stride]; elements past the head dimension are padding."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # the two conditions of one image with guidance, heads of the B shape
        dict(name="packed two conditions", op="packed", dtype="bf16", batch=2, tokens=120, heads=12, kv_heads=12, dim=64, causal=True,
             ragged=True),
        # prompts of different lengths that arrive together, four query heads to a key head
        dict(name="packed ragged prompts", op="packed", dtype="bf16", batch=48, tokens=1144, heads=32, kv_heads=8, dim=128, causal=True,
             ragged=True),
        # one long prompt
        dict(name="packed long prompt", op="packed", dtype="bf16", batch=1, tokens=16384, heads=16, kv_heads=4, dim=128, causal=True,
             ragged=False),
        # earlier frames whose tokens see each other both ways, the 100-element heads of the 3B-shaped stack
        dict(name="packed both ways", op="packed", dtype="f16", batch=4, tokens=2424, heads=32, kv_heads=32, dim=100, causal=False,
             ragged=True),
        # a decode step of the XL shape whose rows have caches of their own
        dict(name="chunk single tokens", op="chunk", dtype="bf16", groups=0, batch=32, new=1, have=1143, prefix=0, heads=20, kv_heads=20,
             dim=64, page=64, ragged=False),
        # a few guessed tokens at a time, checked over long caches
        dict(name="chunk few tokens", op="chunk", dtype="bf16", groups=0, batch=8, new=5, have=16384, prefix=0, heads=32, kv_heads=8,
             dim=128, page=64, ragged=True),
        # the next part of one long prompt
        dict(name="chunk of a long prompt", op="chunk", dtype="f16", groups=0, batch=1, new=1024, have=15360, prefix=0, heads=32,
             kv_heads=8, dim=128, page=64, ragged=False),
        # a row of the grid given for each of 32 batch rows (16 images with guidance) behind the prompt they share
        dict(name="chunk under a prompt", op="chunk", dtype="bf16", groups=2, batch=32, new=32, have=512, prefix=120, heads=20,
             kv_heads=20, dim=64, page=64, ragged=True),
        # the next token of one image
        dict(name="sample one image", op="sample", dtype="bf16", rows=1, vocab=16384, guided=True, top_k=2000, top_p=0.95, min_p=0.0,
             mixed=False),
        # 16 images with guidance
        dict(name="sample sixteen images", op="sample", dtype="bf16", rows=16, vocab=16384, guided=True, top_k=2000, top_p=1.0, min_p=0.0,
             mixed=False),
        # a batch of requests with settings of their own, a large vocabulary
        dict(name="sample large vocabulary", op="sample", dtype="bf16", rows=256, vocab=131072, guided=False, top_k=0, top_p=0.95,
             min_p=0.01, mixed=True),
        # logits in 32 bits, rows of an odd length, few candidates
        dict(name="sample few candidates", op="sample", dtype="f32", rows=64, vocab=50001, guided=False, top_k=50, top_p=0.9, min_p=0.0,
             mixed=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("packed", "chunk", "sample"))
    if op == "sample":
        rows = _log(rng, 1, 256)
        return dict(op=op, dtype=rng.choice(("bf16", "bf16", "f16", "f32")), rows=rows, vocab=_log(rng, 1000, min(131072, 131072 * 128 // rows)),
                    guided=rng.random() < 0.4, top_k=rng.choice((0, 0, 1, 50, 2000)), top_p=rng.choice((1.0, 0.95, 0.9, 0.5)),
                    min_p=rng.choice((0.0, 0.0, 0.02, 0.1)), mixed=rng.random() < 0.5)
    dtype = rng.choice(("bf16", "bf16", "f16"))
    dim = rng.choice((64, 100, 128))
    kv = rng.choice((1, 4, 8, 12, 20))
    heads = kv * rng.choice((1, 1, 2, 4, 8))
    shape = dict(dtype=dtype, heads=heads, kv_heads=kv, dim=dim, ragged=rng.random() < 0.6)
    if op == "packed":
        batch = _log(rng, 1, 48)
        most = int(math.sqrt(16 * 16384 ** 2 / 2 / (heads * batch)))           # (heads * batch * tokens^2 of the long prompt, halved)
        return dict(op=op, batch=batch, tokens=_log(rng, 1, min(16384, most)), causal=rng.random() < 0.8, **shape)
    groups = rng.choice((0, 0, 1, 2))
    batch = max(1, groups) * _log(rng, 1, 32 // max(1, groups))
    new = rng.choice((1, _log(rng, 1, 16), _log(rng, 1, max(1, 4096 // batch))))
    have = _log(rng, 1, max(64, min(16384, 2 ** 31 // (batch * new * heads), 2 ** 27 // (batch * kv * dim)))) - 1
    return dict(op=op, groups=groups, batch=batch, new=new, have=have, prefix=_log(rng, 1, 2424) if groups else 0,
                page=rng.choice((16, 32, 48, 64, 64, 128, 256, 572)), **shape)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _lengths(gen, batch, most, ragged):
    """All alike, or spread evenly from an eighth of `most` to `most` in random order (so that sums do not vary)."""
    if not ragged:
        return torch.full((batch,), most, dtype=torch.int32, device="cuda")
    spread = torch.linspace(max(1, most // 8), most, batch, dtype=torch.float64, device="cuda").round().to(torch.int32)
    return spread[torch.randperm(batch, generator=gen, device="cuda")]


def _starts(lengths):
    return torch.cat([torch.zeros_like(lengths[:1]), lengths.cumsum(0).to(torch.int32)])


def _tables(gen, counts, first=0):
    """Page tables [len(counts)][most], the pages in random order; entries past a row's pages are never read."""
    most = max(1, max(counts))
    order = torch.randperm(sum(counts), generator=gen, device="cuda").to(torch.int32) + first
    table = torch.zeros((len(counts), most), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at:at + n]
        at += n
    return table


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "packed":
        H, KV, d = case["heads"], case["kv_heads"], case["dim"]
        s["cu"] = _starts(_lengths(gen, case["batch"], case["tokens"], case["ragged"]))
        T = int(s["cu"][-1])
        s["q"], s["k"], s["v"] = _normal(gen, (T, H, d), dt, 1.5), _normal(gen, (T, KV, d), dt), _normal(gen, (T, KV, d), dt)
        s["out"] = torch.empty_like(s["q"])
    elif case["op"] == "chunk":
        B, H, KV, d, page = (case[n] for n in ("batch", "heads", "kv_heads", "dim", "page"))
        new = _lengths(gen, B, case["new"], case["ragged"])
        have = _lengths(gen, B, case["have"], case["ragged"]) if case["have"] else torch.zeros_like(new)
        s["n_rows"] = new + have
        s["cu"] = _starts(new)
        T = int(s["cu"][-1])
        counts = [(int(n) + page - 1) // page for n in s["n_rows"].tolist()]
        p_counts = [(case["prefix"] + page - 1) // page] * case["groups"]
        pools = torch.zeros((2, sum(counts) + sum(p_counts), KV, page, (d + 7) // 8 * 8), dtype=dt, device="cuda")
        pools[..., :d].normal_(generator=gen)
        s["k_pool"], s["v_pool"] = pools[0], pools[1]
        s["table"] = _tables(gen, counts)
        s["p_table"] = s["p_rows"] = s["start"] = None
        if case["groups"]:
            s["p_table"] = _tables(gen, p_counts, sum(counts))
            s["p_rows"] = torch.full((case["groups"],), case["prefix"], dtype=torch.int32, device="cuda")
            s["start"] = torch.arange(0, B + 1, B // case["groups"], dtype=torch.int32, device="cuda")
        s["q"] = _normal(gen, (T, H, d), dt, 1.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((T, H), dtype=torch.float32, device="cuda")
    else:
        R, V = case["rows"], case["vocab"]
        # few ids stand out of the many, as a trained model's do
        logits = torch.randn((R, V), generator=gen, device="cuda").mul_(2)
        logits += 4 * (torch.rand((R, V), generator=gen, device="cuda") > 0.999)
        s["uncond"] = None
        if case["guided"]:
            s["uncond"] = logits.to(dt)
            logits = logits + 0.3 * torch.randn((R, V), generator=gen, device="cuda")
        s["logits"] = logits.to(dt)
        s["u"] = torch.rand(R, generator=gen, device="cuda")
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = 0.9, case["top_k"], case["top_p"], case["min_p"]
        if case["mixed"]:                        # each request has its own
            t = torch.rand((3, R), generator=gen, device="cuda")
            s["temperature"] = 0.5 + t[0]
            s["top_k"] = (case["top_k"] * (0.5 + t[1])).ceil().to(torch.int32)
            s["top_p"] = 1 - (1 - case["top_p"]) * 2 * t[2]
            s["min_p"] = torch.full((R,), case["min_p"], device="cuda")
        s["tokens"] = torch.empty(R, dtype=torch.int32, device="cuda")
        s["logprobs"] = torch.empty(R, dtype=torch.float32, device="cuda")
    if own:
        import paper_2506_18226_b200 as A
        s["lib"] = A
        if case["op"] != "sample":
            s["workspace"] = A.prompt_workspace(s["q"], case["kv_heads"], case["batch"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        A = s["lib"]
        if op == "packed":
            return A.packed_attn(s["q"], s["k"], s["v"], s["cu"], causal=s["case"]["causal"], out=s["out"], workspace=s["workspace"])
        if op == "chunk":
            A.chunk_attn(s["q"], s["k_pool"], s["v_pool"], s["table"], s["n_rows"], s["cu"], s["p_table"], s["p_rows"], s["start"],
                         out=s["out"], lse=s["lse"], workspace=s["workspace"])
            return s["out"], s["lse"]
        A.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                 uncond=s["uncond"], guidance=4.0, tokens=s["tokens"], logprobs=s["logprobs"])
        return s["tokens"], s["logprobs"]
    if op == "packed":
        return _plain_packed(s)
    if op == "chunk":
        return _plain_chunk(s)
    return _plain_sample(s)


def _softmax_product(q, k, v, seen):
    """q [.., T, KV, g, d], k and v [.., KV, R, d], seen [.., T, R] -> out like q, ln sum exp [.., T, KV, g], all in 32 bits."""
    B, T, KV, g, d = q.shape
    logits = q.permute(0, 2, 3, 1, 4).reshape(B, KV, g * T, d) @ k.transpose(-1, -2)
    logits = logits.view(B, KV, g, T, -1).masked_fill_(~seen[:, None, None], -math.inf)
    most = logits.amax(-1, keepdim=True)
    weight = logits.sub_(most).exp_()
    total = weight.sum(-1, keepdim=True)
    out = (weight.view(B, KV, g * T, -1) @ v).view(B, KV, g, T, d) / total
    return out.permute(0, 3, 1, 2, 4), (most + total.log())[..., 0].permute(0, 3, 1, 2)


def _spread(x, cu, most):
    """Tokens laid end to end -> [batch, most, ..] (what stands past a sequence's end is any token)."""
    at = cu[:-1, None] + torch.arange(most, device="cuda")
    return x[at.clamp(max=x.shape[0] - 1)]


def _gathered(x, cu, tokens):
    """The inverse: the tokens of every sequence out of [batch, most, ..]."""
    t = torch.arange(tokens, device="cuda")
    b = torch.bucketize(t, cu[1:], right=True)
    return x[b, t - cu[b]]


def _plain_packed(s):
    c = s["case"]
    T, KV, d = c["tokens"], c["kv_heads"], c["dim"]
    q, k, v = (_spread(s[n], s["cu"], T).float() for n in "qkv")
    at = torch.arange(T, device="cuda")
    seen = (at < (s["cu"][1:] - s["cu"][:-1])[:, None])[:, None, :].expand(-1, T, -1)
    if c["causal"]:
        seen = seen & (at <= at[:, None])
    out, _ = _softmax_product(q.unflatten(2, (KV, -1)) / math.sqrt(d), k.transpose(1, 2), v.transpose(1, 2), seen)
    return _gathered(out, s["cu"], s["q"].shape[0]).flatten(1, 2).to(s["q"].dtype)


def _plain_chunk(s):
    c = s["case"]
    B, T, KV, d = c["batch"], c["new"], c["kv_heads"], c["dim"]

    def rows(pool, table):                       # [n][pages] -> [n][KV][rows][d]
        return pool[table.long()][..., :d].transpose(1, 2).reshape(table.shape[0], KV, -1, d).float()

    k, v = rows(s["k_pool"], s["table"]), rows(s["v_pool"], s["table"])
    new = s["cu"][1:] - s["cu"][:-1]
    last = (s["n_rows"] - new)[:, None] + torch.arange(T, device="cuda")          # the row that each new token is
    seen = torch.arange(k.shape[2], device="cuda") <= last[..., None]
    if c["groups"]:
        g = torch.bucketize(torch.arange(B, device="cuda"), s["start"][1:], right=True)
        pk, pv = rows(s["k_pool"], s["p_table"])[g], rows(s["v_pool"], s["p_table"])[g]
        before = torch.arange(pk.shape[2], device="cuda") < s["p_rows"][g][:, None]
        k, v = torch.cat([pk, k], 2), torch.cat([pv, v], 2)
        seen = torch.cat([before[:, None].expand(-1, T, -1), seen], 2)
    q = _spread(s["q"], s["cu"], T).float().unflatten(2, (KV, -1)) / math.sqrt(d)
    out, lse = _softmax_product(q, k, v, seen)
    n = s["q"].shape[0]
    return _gathered(out, s["cu"], n).flatten(1, 2).to(s["q"].dtype), _gathered(lse, s["cu"], n).flatten(1)


def _per_row(x, rows, dtype):
    return (x if torch.is_tensor(x) else torch.full((rows,), x, device="cuda")).to(dtype)[:, None]


def _plain_sample(s):
    """Logits as they are, or mixed in 32 bits; weights and their sums in 64, since an id is kept or drawn by a comparison."""
    x = s["logits"].float()
    R, V = x.shape
    if s["uncond"] is not None:
        u = s["uncond"].float()
        x = u + 4.0 * (x - u)
    temperature, top_p, min_p = (_per_row(s[n], R, torch.float32).double() for n in ("temperature", "top_p", "min_p"))
    top_k = _per_row(s["top_k"], R, torch.int64)
    x, order = x.sort(dim=-1, descending=True, stable=True)                           # equal logits: the lower id first
    z = (x.double() - x[:, :1].double()) / temperature
    weight = z.exp()
    kept = (top_k <= 0) | (torch.arange(V, device="cuda") < top_k)
    mass = torch.where(kept, weight, 0.0)
    before = mass.cumsum(-1) - mass
    kept &= (top_p >= 1) | (before < top_p * mass.sum(-1, keepdim=True))
    kept &= weight >= min_p
    mass = torch.where(kept, weight, 0.0)
    total = mass.sum(-1, keepdim=True)
    by_id = torch.zeros_like(mass).scatter_(1, order, mass)
    kept_by_id = torch.zeros_like(kept).scatter_(1, order, kept)
    reached = kept_by_id & (by_id.cumsum(-1) >= s["u"][:, None].double() * total)
    token = reached.to(torch.int8).argmax(-1, keepdim=True)
    logprob = torch.zeros_like(z).scatter_(1, order, z).gather(1, token) - total.log()
    return token[:, 0].to(torch.int32), logprob[:, 0].float()


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def _spread_lengths(count, most, ragged):
    low = max(1, most // 8)
    return [most if not ragged else low + (most - low) * i / max(1, count - 1) for i in range(count)]


def work(case):
    c = case
    if c["op"] == "sample":
        n = c["rows"] * c["vocab"] * (2 if c["guided"] else 1)
        return {"bytes": n * (4 if c["dtype"] == "f32" else 2) + 12 * c["rows"], "flops": 4 * n}
    pair = 4 * c["heads"] * c["dim"]
    if c["op"] == "packed":
        n = _spread_lengths(c["batch"], c["tokens"], c["ragged"])
        pairs = sum(x * (x + 1) / 2 if c["causal"] else x * x for x in n)
        return {"bytes": 4 * sum(n) * c["dim"] * (c["heads"] + c["kv_heads"]), "flops": pair * pairs}
    new = _spread_lengths(c["batch"], c["new"], c["ragged"])
    have = _spread_lengths(c["batch"], c["have"], c["ragged"]) if c["have"] else [0] * c["batch"]
    mean = sum(have) / c["batch"]
    rows = sum(new) + sum(have) + c["groups"] * c["prefix"]
    pairs = sum(x * (c["prefix"] + mean) + x * (x + 1) / 2 for x in new)
    return {"bytes": rows * c["kv_heads"] * c["dim"] * 4 + sum(new) * c["heads"] * (4 * c["dim"] + 4), "flops": pair * pairs}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_heads(q, k, v, seen):
    """q [T][H][d], k and v [R][KV][d], seen [T][R] (None: all) -> out [T][H][d], lse [T][H], a key head at a time."""
    H, KV, d = q.shape[1], k.shape[1], q.shape[2]
    out, lse = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    for h in range(H):
        key, value = k[:, h * KV // H].double(), v[:, h * KV // H].double()
        logits = (q[:, h].double() @ key.T).div_(math.sqrt(d))
        if seen is not None:
            logits.masked_fill_(~seen, -math.inf)
        out[:, h] = torch.softmax(logits, 1) @ value
        lse[:, h] = torch.logsumexp(logits, 1)
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "packed":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        cu = s["cu"].tolist()
        for a, b in zip(cu, cu[1:]):
            seen = torch.ones((b - a, b - a), dtype=torch.bool, device="cuda").tril_() if case["causal"] else None
            out[a:b] = _exact_heads(s["q"][a:b], s["k"][a:b], s["v"][a:b], seen)[0]
        return out
    if case["op"] == "chunk":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
        cu, n_rows, d, page = s["cu"].tolist(), s["n_rows"].tolist(), case["dim"], case["page"]

        def rows(pool, table, n):                # [n][KV][d]
            at = torch.arange(n, device="cuda")
            return pool[table[at // page].long(), :, at % page, :d]

        for b in range(case["batch"]):
            m, n, p = cu[b + 1] - cu[b], n_rows[b], case["prefix"]
            k, v = rows(s["k_pool"], s["table"][b], n), rows(s["v_pool"], s["table"][b], n)
            if p:
                t = s["p_table"][b * case["groups"] // case["batch"]]
                k, v = torch.cat([rows(s["k_pool"], t, p), k]), torch.cat([rows(s["v_pool"], t, p), v])
            seen = torch.ones((m, p + n), dtype=torch.bool, device="cuda").tril_(p + n - m)
            out[cu[b]:cu[b + 1]], lse[cu[b]:cu[b + 1]] = _exact_heads(s["q"][cu[b]:cu[b + 1]], k, v, seen)
        return out, lse
    logprobs = torch.empty(case["rows"], dtype=torch.float64, device="cuda")
    for r in range(case["rows"]):
        T, k, p, least = (float(x[r] if torch.is_tensor(x) else torch.tensor(x, dtype=torch.float32)) for x in
                          (s["temperature"], s["top_k"], s["top_p"], s["min_p"]))
        x = s["logits"][r].float()
        if case["guided"]:
            x = s["uncond"][r].float() + 4.0 * (x - s["uncond"][r].float())
        prob = torch.softmax(x.double() / T, 0)
        ids = torch.argsort(-x.double(), stable=True)
        if k > 0:
            ids = ids[:int(k)]
        if p < 1:
            share = prob[ids].cumsum(0)
            ids = ids[:int((share < p * share[-1]).sum()) + 1]
        ids = ids[prob[ids] >= least * prob[ids[0]]].sort().values
        share = prob[ids].cumsum(0)
        i = min(int((share < float(s["u"][r]) * share[-1]).sum()), len(ids) - 1)
        logprobs[r] = prob[ids[i]].log() - share[-1].log()
    return None, logprobs
