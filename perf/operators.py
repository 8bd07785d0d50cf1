"""Cases, inputs, plain forms and exact values for the operators of a decoder that makes many images of one prompt:
rotary positions with several axes, the rotated append into a paged cache, decode attention over a shared prefix, and the
norms around a block with its gate and residual scale.

A pool is [n_pages][n_kv_heads][page_rows][row_stride]; elements past the head dimension are padding (zero)."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# pairs of elements that turn with each axis, by head dimension and number of axes
PAIRS = {(64, 1): (32,), (64, 2): (16, 16), (64, 3): (8, 12, 12), (100, 2): (25, 25), (100, 3): (10, 20, 20),
         (128, 1): (64,), (128, 2): (32, 32), (128, 3): (16, 24, 24)}


def listed():
    return [
        # the queries of one decode step of the XL shape: 32 batch rows, grid row and column
        dict(name="rope decode step", op="rope", dtype="bf16", tokens=32, heads=20, dim=64, axes=2, halves=False, restart=True,
             packed=False, origin=0),
        # a clip of eight 48 x 48 frames, deep into a long session, out of a packed q/k/v projection
        dict(name="rope video prompt", op="rope", dtype="bf16", tokens=18432, heads=32, dim=128, axes=3, halves=True,
             restart=False, packed=True, origin=1000000),
        # the 100-element heads of the 3B-shaped stack, one prompt and its grid
        dict(name="rope wide heads", op="rope", dtype="f16", tokens=2424, heads=32, dim=100, axes=3, halves=False, restart=True,
             packed=False, origin=0),
        # one decode step of the XL shape: a row per stream, q turned on the way
        dict(name="append decode step", op="append", dtype="bf16", batch=32, kv_heads=20, q_heads=20, dim=64, axes=2,
             halves=False, restart=True, page=64, new=1, have=1023, ragged=False),
        # prompts of different lengths entering an empty cache, four query heads to a key head
        dict(name="append ragged prompts", op="append", dtype="bf16", batch=48, kv_heads=8, q_heads=32, dim=128, axes=3,
             halves=True, restart=False, page=64, new=1144, have=0, ragged=True),
        # a few tokens at once on 100-element heads, pages that are no power of two
        dict(name="append wide heads", op="append", dtype="f16", batch=64, kv_heads=32, q_heads=0, dim=100, axes=2,
             halves=False, restart=True, page=48, new=17, have=700, ragged=True),
        # one decode step of the XL shape
        dict(name="norm decode step", op="norm", dtype="bf16", rows=32, dim=1280, post=True, gates=32, wide=False),
        # the condition and grid of 32 batch rows, gates per batch row, residual stream kept in 32 bits
        dict(name="norm prompts", op="norm", dtype="bf16", rows=36608, dim=1280, post=True, gates=32, wide=True),
        # one image with guidance, early in its grid
        dict(name="attn one image", op="attn", dtype="bf16", groups=2, members=1, heads=12, kv_heads=12, dim=64, prefix=120,
             own_rows=100, page=64, ragged=False),
        # 16 images of one prompt with guidance, at the end of a 32 x 32 grid
        dict(name="attn sixteen images", op="attn", dtype="bf16", groups=2, members=16, heads=20, kv_heads=20, dim=64,
             prefix=120, own_rows=1024, page=64, ragged=False),
        # 64 continuations of one long context of earlier images, four query heads to a key head
        dict(name="attn long context", op="attn", dtype="bf16", groups=1, members=64, heads=32, kv_heads=8, dim=128,
             prefix=32768, own_rows=1024, page=64, ragged=True),
        # four prompts with an earlier frame each, 100-element heads, pages that are no power of two
        dict(name="attn wide heads", op="attn", dtype="f16", groups=4, members=16, heads=32, kv_heads=32, dim=100,
             prefix=2424, own_rows=2304, page=48, ragged=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rope", "append", "norm", "attn", "attn"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "norm":
        dim = 8 * _log(rng, 12, 512)
        gates = rng.choice((0, 1, 2, 16, 32))
        n = max(1, gates)
        rows = n * _log(rng, 1, max(1, 36608 * 1280 // (dim * n)))
        return dict(op=op, dtype=dtype, rows=rows, dim=dim, post=rng.random() < 0.7, gates=gates, wide=rng.random() < 0.4)
    dim, axes = rng.choice(sorted(PAIRS))
    turn = dict(dim=dim, axes=axes, halves=rng.random() < 0.5, restart=rng.random() < 0.5)
    if op == "rope":
        heads = rng.choice((1, 8, 12, 20, 32))
        return dict(op=op, dtype=dtype, tokens=_log(rng, 1, 18432 * 32 * 128 // (heads * dim) // 2), heads=heads, **turn,
                    packed=rng.random() < 0.5, origin=rng.choice((0, 5000, 1000000)))
    page = rng.choice((16, 32, 48, 64, 64, 128, 256, 572))
    if op == "append":
        kv = rng.choice((1, 4, 8, 20))
        batch = _log(rng, 1, 64)
        return dict(op=op, dtype=dtype, batch=batch, kv_heads=kv, q_heads=kv * rng.choice((0, 1, 4)), **turn, page=page,
                    new=rng.choice((1, _log(rng, 1, 1144))), have=_log(rng, 1, 1500) - 1, ragged=rng.random() < 0.5)
    groups = rng.choice((1, 2, 2, 4))
    members = _log(rng, 1, 64 // groups)
    kv = rng.choice((1, 4, 8, 12, 20))
    heads = kv * rng.choice((1, 1, 2, 4, 8))
    queries = groups * members * heads
    prefix = _log(rng, 1, max(64, min(32768, 32768 * 2048 // (queries * groups))))
    return dict(op=op, dtype=dtype, groups=groups, members=members, heads=heads, kv_heads=kv, dim=dim, prefix=prefix,
                own_rows=_log(rng, 1, 2304), page=page, ragged=rng.random() < 0.6)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _pool(gen, pages, heads, page, dim, dtype):
    """Rows with padding to a multiple of eight elements."""
    pool = torch.zeros((pages, heads, page, (dim + 7) // 8 * 8), dtype=dtype, device="cuda")
    pool[..., :dim].normal_(generator=gen)
    return pool


def _lengths(gen, batch, most, ragged):
    """All alike, or spread evenly from an eighth of `most` to `most` in random order (so that sums do not vary)."""
    if not ragged:
        return torch.full((batch,), most, dtype=torch.int32, device="cuda")
    spread = torch.linspace(max(1, most // 8), most, batch, dtype=torch.float64, device="cuda").round().to(torch.int32)
    return spread[torch.randperm(batch, generator=gen, device="cuda")]


def _positions(tokens, axes, origin):
    """Raster order over frames of 48 x 48; one axis: the index; two: row and column; three: frame, row, column."""
    t = torch.arange(tokens, device="cuda")
    cols = {1: (t + origin,), 2: (t // 48 + origin, t % 48), 3: (t // 2304 + origin, t // 48 % 48, t % 48)}[axes]
    return torch.stack(cols, 1).to(torch.int32).contiguous()


def _tables(gen, counts, first=0, pages=0):
    """Page tables [len(counts)][most], a random choice of pages; entries past a row's pages are never read."""
    most = max(1, max(counts))
    order = torch.randperm(max(pages, sum(counts)), generator=gen, device="cuda").to(torch.int32) + first
    table = torch.zeros((len(counts), most), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at:at + n]
        at += n
    return table


def prepare(case, seed):
    gen = _generator(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "rope":
        T, H, d = case["tokens"], case["heads"], case["dim"]
        if case["packed"]:                       # q of a packed [q, k, v] projection
            s["x"] = _normal(gen, (T, 3, H, d), dt)[:, 0]
        else:
            s["x"] = _normal(gen, (T, H, d), dt)
        s["pos"] = _positions(T, case["axes"], case["origin"])
        s["out"] = torch.empty((T, H, d), dtype=dt, device="cuda")
    elif case["op"] == "append":
        B, KV, QH, d, page = case["batch"], case["kv_heads"], case["q_heads"], case["dim"], case["page"]
        new = _lengths(gen, B, case["new"], case["ragged"])
        have = _lengths(gen, B, case["have"], case["ragged"]) if case["have"] else torch.zeros_like(new)
        counts = [(int(n) + page - 1) // page for n in (new + have).tolist()]
        pages = sum(int(n) // page + 2 for n in new.tolist()) + sum(int(n) // page for n in have.tolist())
        T = int(new.sum())
        s["k"], s["v"] = _normal(gen, (T, KV, d), dt), _normal(gen, (T, KV, d), dt)
        s["q"] = _normal(gen, (T, QH, d), dt) if QH else None
        s["q_out"] = torch.empty_like(s["q"]) if QH else None
        s["table"] = _tables(gen, counts, pages=pages)
        s["n_rows"] = have
        s["cu"] = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0).to(torch.int32)]) if case["ragged"] else None
        s["pos"] = _positions(T, case["axes"], 7)
        s["k_pool"], s["v_pool"] = (torch.zeros((pages, KV, page, (d + 7) // 8 * 8), dtype=dt, device="cuda") for _ in range(2))
    elif case["op"] == "norm":
        R, D = case["rows"], case["dim"]
        s["y"] = _normal(gen, (R, D), dt, 0.7)
        s["x"] = _normal(gen, (R, D), torch.float32 if case["wide"] else dt, 2.0)
        s["w_pre"] = (1 + 0.1 * torch.randn(D, generator=gen, device="cuda")).to(dt)
        s["w_post"] = (1 + 0.1 * torch.randn(D, generator=gen, device="cuda")).to(dt) if case["post"] else None
        s["gate"] = _normal(gen, (case["gates"], D), dt, 0.5) if case["gates"] else None
        s["x_out"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["y"])
    else:
        G, M, H, KV, d, page = (case[n] for n in ("groups", "members", "heads", "kv_heads", "dim", "page"))
        B = G * M
        n_rows = _lengths(gen, B, case["own_rows"], case["ragged"])
        p_rows = _lengths(gen, G, case["prefix"], False)
        counts = [(int(n) + page - 1) // page for n in n_rows.tolist()]
        p_counts = [(case["prefix"] + page - 1) // page] * G
        s["k_pool"], s["v_pool"] = (_pool(gen, sum(counts) + sum(p_counts), KV, page, d, dt) for _ in range(2))
        s["table"], s["n_rows"] = _tables(gen, counts), n_rows
        s["p_table"], s["p_rows"] = _tables(gen, p_counts, sum(counts)), p_rows
        s["start"] = torch.arange(0, B + 1, M, dtype=torch.int32, device="cuda")
        s["q"] = _normal(gen, (B, H, d), dt, 1.5)
        s["out"] = torch.empty((B, H, d), dtype=dt, device="cuda")
        s["lse"] = torch.empty((B, H), dtype=torch.float32, device="cuda")
    if own:
        import paper_2506_18226_b200 as A
        s["lib"] = A
        if case["op"] in ("rope", "append"):
            s["rotary"] = A.Rotary(case["dim"], PAIRS[case["dim"], case["axes"]], style="halves" if case["halves"] else "pairs",
                                   restart=case["restart"])
        if case["op"] == "attn":
            s["workspace"] = A.shared_prefix_workspace(s["q"], s["k_pool"], s["table"], s["p_table"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        A = s["lib"]
        if op == "rope":
            return A.rope_axes(s["rotary"], s["x"], s["pos"], out=s["out"])
        if op == "append":
            A.paged_append(s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"], s["n_rows"], cu_tokens=s["cu"],
                           rotary=s["rotary"], pos=s["pos"], q=s["q"], q_out=s["q_out"])
            return s["q_out"], s["k_pool"], s["v_pool"]
        if op == "norm":
            return A.norm_residual(s["y"], s["x"], s["w_pre"], w_post=s["w_post"], gate=s["gate"], scale=0.5, eps=1e-5,
                                   x_out=s["x_out"], h=s["h"])
        A.shared_prefix_attn(s["q"], s["k_pool"], s["v_pool"], s["table"], s["n_rows"], s["p_table"], s["p_rows"], s["start"],
                             out=s["out"], lse=s["lse"], workspace=s["workspace"])
        return s["out"], s["lse"]
    if op == "rope":
        return _plain_turn(s["case"], s["x"], s["pos"])
    if op == "append":
        return _plain_append(s)
    if op == "norm":
        return _plain_norm(s)
    return _plain_attn(s)


def _plain_turn(case, x, pos):
    """Angles in 64 bits (a far position times a frequency loses the turn in 32), the rotation in 32."""
    pairs = PAIRS[case["dim"], case["axes"]]
    n, d = sum(pairs), case["dim"]
    sizes = torch.tensor(pairs, device=x.device)
    axis = torch.repeat_interleave(torch.arange(len(pairs), device=x.device), sizes, output_size=n)
    i = torch.arange(n, device=x.device)
    if case["restart"]:
        i = i - (torch.cumsum(sizes, 0) - sizes)[axis]
        freq = torch.pow(10000.0, -i.double() / sizes[axis])
    else:
        freq = torch.pow(10000.0, -i.double() / n)
    angle = pos[:, axis].double() * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    a, b = (x[..., :n], x[..., n:2 * n]) if case["halves"] else (x[..., 0:2 * n:2], x[..., 1:2 * n:2])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([ra, rb], -1) if case["halves"] else torch.stack([ra, rb], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * n:d]], -1).to(DTYPES[case["dtype"]])


def _plain_append(s):
    c = s["case"]
    T, d = s["k"].shape[0], c["dim"]
    t = torch.arange(T, device="cuda")
    if s["cu"] is None:
        b, j = t // c["new"], t % c["new"]
    else:
        b = torch.bucketize(t, s["cu"][1:], right=True)
        j = t - s["cu"][b]
    row = s["n_rows"][b] + j
    page = s["table"][b, row // c["page"]].long()
    s["k_pool"][page, :, row % c["page"], :d] = _plain_turn(c, s["k"], s["pos"])
    s["v_pool"][page, :, row % c["page"], :d] = s["v"]
    if s["q"] is not None:
        s["q_out"] = _plain_turn(c, s["q"], s["pos"])
    return s["q_out"], s["k_pool"], s["v_pool"]


def _plain_norm(s):
    eps = 1e-5
    z, x = s["y"].float(), s["x"].float()
    if s["w_post"] is not None:
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps) * s["w_post"].float()
    if s["gate"] is not None:
        n = s["gate"].shape[0]
        z = (z.view(n, -1, z.shape[-1]) * s["gate"].float()[:, None]).view_as(z)
    x = x + 0.5 * z
    h = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * s["w_pre"].float()
    return x.to(s["x"].dtype), h.to(s["y"].dtype)


def _plain_attn(s):
    c = s["case"]
    G, M, H, KV, d = (c[n] for n in ("groups", "members", "heads", "kv_heads", "dim"))
    B, g = G * M, H // KV

    def gather(pool, table):                     # [n][pages] -> [n][KV][rows][d] in 32 bits
        return pool[table.long()][..., :d].transpose(1, 2).reshape(table.shape[0], KV, -1, d).float()

    q = s["q"].float() / math.sqrt(d)
    # the prefix: every group's queries of a key head in one product
    kp, vp = gather(s["k_pool"], s["p_table"]), gather(s["v_pool"], s["p_table"])
    qp = q.view(G, M, KV, g, d).transpose(1, 2).reshape(G, KV, M * g, d)
    sp = qp @ kp.transpose(-1, -2)
    sp = sp.masked_fill(torch.arange(sp.shape[-1], device="cuda") >= s["p_rows"][:, None, None, None], -math.inf)
    mp = sp.amax(-1, keepdim=True)
    ep = torch.exp(sp - mp)
    op, lp = ep @ vp, ep.sum(-1, keepdim=True)
    op, lp, mp = (x.view(G, KV, M, g, -1).transpose(1, 2).reshape(B, KV, g, -1) for x in (op, lp, mp))
    # each batch row's own rows
    kr, vr = gather(s["k_pool"], s["table"]), gather(s["v_pool"], s["table"])
    sr = q.view(B, KV, g, d) @ kr.transpose(-1, -2)
    sr = sr.masked_fill(torch.arange(sr.shape[-1], device="cuda") >= s["n_rows"][:, None, None, None], -math.inf)
    mr = sr.amax(-1, keepdim=True)
    er = torch.exp(sr - mr)
    orow, lr = er @ vr, er.sum(-1, keepdim=True)
    m = torch.maximum(mp, mr)
    wp, wr = torch.exp(mp - m), torch.exp(mr - m)
    total = wp * lp + wr * lr
    out = (wp * op + wr * orow) / total
    return out.reshape(B, H, d).to(DTYPES[c["dtype"]]), (m + torch.log(total)).reshape(B, H)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def _ragged_mean(most, ragged):
    return (max(1, most // 8) + most) / 2 if ragged else most


def work(case):
    c = case
    if c["op"] == "rope":
        n = c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": 4 * n + 4 * c["tokens"] * c["axes"], "flops": 3 * n}
    if c["op"] == "append":
        tokens = c["batch"] * _ragged_mean(c["new"], c["ragged"])
        n = tokens * (2 * c["kv_heads"] + c["q_heads"]) * c["dim"]
        return {"bytes": 4 * n + 4 * tokens * c["axes"], "flops": 3 * tokens * (c["kv_heads"] + c["q_heads"]) * c["dim"]}
    if c["op"] == "norm":
        n, x = c["rows"] * c["dim"], 4 if c["wide"] else 2
        return {"bytes": n * (4 + 2 * x) + 2 * c["dim"] * (2 + c["gates"]), "flops": 10 * n}
    B = c["groups"] * c["members"]
    own_rows = _ragged_mean(c["own_rows"], c["ragged"])
    rows = c["groups"] * c["prefix"] + B * own_rows
    return {"bytes": rows * c["kv_heads"] * c["dim"] * 4 + B * c["heads"] * (4 * c["dim"] + 4),
            "flops": 4 * B * c["heads"] * c["dim"] * (c["prefix"] + own_rows)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_turn(case, x, pos):
    """A pair is a complex number, turned by exp(i * position * frequency)."""
    pairs = PAIRS[case["dim"], case["axes"]]
    n = sum(pairs)
    turn = []
    for a, count in enumerate(pairs):
        for j in range(count):
            exponent = j / count if case["restart"] else len(turn) / n
            turn.append(pos[:, a].double() * 10000.0 ** -exponent)
    angle = torch.stack(turn, 1)
    z = x.double()
    if case["halves"]:
        z = z[..., :2 * n].unflatten(-1, (2, n)).transpose(-1, -2)
    else:
        z = z[..., :2 * n].unflatten(-1, (n, 2))
    z = torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    z = torch.view_as_real(z)
    out = x.double().clone()
    out[..., :2 * n] = (z.transpose(-1, -2) if case["halves"] else z).flatten(-2)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_turn(case, s["x"], s["pos"])
    if case["op"] == "append":
        k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
        k = _exact_turn(case, s["k"], s["pos"])
        first = s["cu"].tolist() if case["ragged"] else list(range(0, s["k"].shape[0] + 1, case["new"]))
        have, table, page = s["n_rows"].tolist(), s["table"].tolist(), case["page"]
        for b in range(case["batch"]):
            i = first[b]
            while i < first[b + 1]:              # one page after another
                row = have[b] + i - first[b]
                n = min(page - row % page, first[b + 1] - i)
                for pool, rows in ((k_pool, k), (v_pool, s["v"])):
                    pool[table[b][row // page], :, row % page:row % page + n, :case["dim"]] = rows[i:i + n].transpose(0, 1).double()
                i += n
        return None if s["q"] is None else _exact_turn(case, s["q"], s["pos"]), k_pool, v_pool
    if case["op"] == "norm":
        z, x = s["y"].double(), s["x"].double()
        if case["post"]:
            z = z * torch.rsqrt(z.square().mean(1, keepdim=True) + 1e-5) * s["w_post"].double()
        if case["gates"]:
            z = z * s["gate"].double().repeat_interleave(case["rows"] // case["gates"], 0)
        x = x + 0.5 * z
        return x, x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5) * s["w_pre"].double()
    B, H, d = s["q"].shape
    KV, page = case["kv_heads"], case["page"]
    out = torch.empty((B, H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, H), dtype=torch.float64, device="cuda")

    def rows(pool, table, n):                    # [KV][n][d]
        at = torch.arange(n, device="cuda")
        return pool[table[at // page].long(), :, at % page, :d].transpose(0, 1).double()

    for g in range(case["groups"]):
        n = int(s["p_rows"][g])
        kp, vp = rows(s["k_pool"], s["p_table"][g], n), rows(s["v_pool"], s["p_table"][g], n)
        for b in range(g * case["members"], (g + 1) * case["members"]):
            n = int(s["n_rows"][b])
            q = s["q"][b].double().view(KV, H // KV, d) / math.sqrt(d)
            k, v = rows(s["k_pool"], s["table"][b], n), rows(s["v_pool"], s["table"][b], n)
            logits = torch.cat([q @ kp.transpose(1, 2), q @ k.transpose(1, 2)], 2)
            weight = torch.softmax(logits, 2)
            out[b] = (weight[..., :kp.shape[1]] @ vp + weight[..., kp.shape[1]:] @ v).view(H, d)
            lse[b] = torch.logsumexp(logits, 2).view(H)
    return out, lse
