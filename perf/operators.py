"""The operators that put several tokens at once into a cache: the norm and position rotation
of queries and keys (written into the cache's rows), the attention of packed prompts, the
attention of a tree of drafted tokens, and the commit of an accepted path.

With ``own`` false every operator is computed in its plain form (elementary torch operations
in float32, angles in float64), with ``own`` true through the framework's entry points.
``exact`` is the same mathematics in float64, sequence by sequence.

Layouts: projections are one [N][(Hq + 2 Hk) D] product, as a fused projection leaves it;
packed tokens of sequence b are cu[b] .. cu[b + 1] - 1; caches are [batch * Hk][capacity][D].
Token r of a sequence belongs in row len + r of its units.
"""
import math

import torch

own = False


def _case(name, kind, **kw):
    c = {"name": name, "kind": kind, "batch": 1, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16",
         "rows": 0, "tokens": 1, "uneven": False}
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of 16 sequences: queries and keys on their way to the decode kernel
        _case("rope_step_b16", "rope", batch=16, cache=False, rot=128, interleaved=False, norm=True, far=16384),
        # the projections of eight packed prompts, about 16k tokens, into the cache
        _case("rope_prompt_b8", "rope", batch=8, tokens=4001, uneven=True, cache=True, rot=128, interleaved=False,
              norm=True, far=0),
        # the toy model's float32 heads, half of each rotated in adjacent pairs, far positions, no norm
        _case("rope_f32_far", "rope", batch=3, kv_heads=2, group=2, head_dim=64, dtype="f32", tokens=700, uneven=True,
              cache=True, rot=32, interleaved=True, norm=False, far=1000000),
        # the toy model's prompt of 512 tokens in float32
        _case("prompt_f32_toy", "prompt", kv_heads=2, group=2, head_dim=64, dtype="f32", tokens=512),
        # a batch of short questions of different lengths
        _case("prompt_short_b16", "prompt", batch=16, tokens=255, uneven=True),
        # prompts of 2k tokens with 64-element heads, eight queries to a key head
        _case("prompt_2k_d64", "prompt", batch=4, group=8, head_dim=64, tokens=2048),
        # the next 512 tokens of one long prompt behind 16k rows that are in the cache
        _case("prompt_chunk_16k", "prompt", rows=16384, tokens=512),
        # two whole 8k prompts of the 32-query-head model: the largest
        _case("prompt_8k_b2", "prompt", batch=2, tokens=8192),
        # a small draft over one sequence's 4k cache: latency
        _case("tree_4k_b1", "tree", rows=4096, tokens=13),
        # 16 sequences of a served batch, 16k rows, up to 32 drafted tokens each
        _case("tree_16k_b16", "tree", batch=16, rows=16384, tokens=32, uneven=True),
        # one speculative step of one sequence: rope, tree attention, commit of the accepted path
        _case("verify_1k_b1", "verify", rows=1024, tokens=8),
        # the same for eight sequences with evicted caches of uneven lengths, 64 drafted tokens each
        _case("verify_8k_b8", "verify", batch=8, rows=8192, tokens=64, uneven=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "prompt", "prompt", "prompt", "tree", "tree", "verify"])
    c = {"kind": kind, "kv_heads": rng.choice([1, 2, 4, 8, 8]), "group": rng.choice([1, 2, 4, 4, 8]),
         "head_dim": rng.choice([64, 128, 128]), "dtype": "f32" if rng.random() < 0.15 else "bf16",
         "uneven": rng.random() < 0.6, "rows": 0}
    if kind == "rope":
        c.update(batch=_log(rng, 1, 16), tokens=_log(rng, 1, 4001), cache=rng.random() < 0.7,
                 rot=rng.choice([c["head_dim"], c["head_dim"], c["head_dim"] // 2, 16]),
                 interleaved=rng.random() < 0.3, norm=rng.random() < 0.7, far=rng.choice([0, 16384, 1000000]),
                 rows=_log(rng, 1, 2048) if rng.random() < 0.5 else 0)
        c["batch"] = max(1, min(c["batch"], 16384 // c["tokens"]))
    elif kind == "prompt":
        c.update(batch=_log(rng, 1, 32), tokens=_log(rng, 1, 8192),
                 rows=_log(rng, 16, 16384) if rng.random() < 0.4 else 0)
        most = 2 * 32 * 8192 * 8192 // (4 if c["dtype"] == "f32" else 1)
        each = c["kv_heads"] * c["group"] * c["tokens"] * (c["tokens"] + c["rows"])
        while each > most:
            c["tokens"] //= 2
            each = c["kv_heads"] * c["group"] * c["tokens"] * (c["tokens"] + c["rows"])
        c["batch"] = max(1, min(c["batch"], most // each, 16384 // c["tokens"]))
    else:
        c.update(batch=_log(rng, 1, 16), tokens=_log(rng, 1, 64), rows=_log(rng, 200, 16384))
        if c["dtype"] == "f32":
            c["batch"] = min(c["batch"], 4)
    return c


# ------------------------------------------------------------------------ sizes

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _counts(c):
    """Tokens of each sequence: all `tokens`, or the first that many and the others fewer."""
    n = c["tokens"]
    if not c["uneven"]:
        return [n] * c["batch"]
    return [max(1, n - (n * ((5 * b) % 8)) // 9) for b in range(c["batch"])]


def _lens(c):
    """Rows of each unit before the call: heads of an evicted cache keep different numbers."""
    u = c["batch"] * c["kv_heads"]
    if not (c["uneven"] and c["kind"] in ("tree", "verify")):
        return [c["rows"]] * u
    return [max(1, c["rows"] - (c["rows"] * ((3 * i) % 7)) // 13) for i in range(u)]


def _keeps(c):
    """Accepted tokens of each sequence: about a quarter of the drafted ones, all equal where the lengths are."""
    n = _counts(c)
    return [max(1, x // 4 + (b % 2 if c["uneven"] and x >= 8 else 0)) for b, x in enumerate(n)]


def work(c):
    n, hk, hq, d = _counts(c), c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"]
    e, total = (4 if c["dtype"] == "f32" else 2), sum(_counts(c))
    rope = {"bytes": 2 * total * (hq + (2 * hk if c["kind"] == "verify" or c.get("cache") else hk)) * d * e,
            "flops": 8 * total * (hq + hk) * d}
    if c["kind"] == "rope":
        return rope
    lens = _lens(c)
    rows = sum(lens) + hk * total
    tree = c["kind"] != "prompt"
    pairs = sum((lens[b * hk] * x + (x * x if tree else x * (x + 1) / 2)) for b, x in enumerate(n)) * hq
    att = {"bytes": 2 * total * hq * d * e + 2 * rows * d * e, "flops": 4 * d * pairs}
    if c["kind"] != "verify":
        return att
    kept = sum(_keeps(c)) * hk
    return {"bytes": rope["bytes"] + att["bytes"] + kept * (4 * d * e + 28), "flops": rope["flops"] + att["flops"]}


# ------------------------------------------------------------------------ inputs

EPS = 1e-6


def _randn(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _key_rows(g, shape, dtype):
    """Key rows with log-normal norms, as the framework's synthetic caches have."""
    return (torch.randn(shape, generator=g, device="cuda")
            * torch.exp(0.5 * torch.randn(shape[:-1], generator=g, device="cuda"))[..., None]).to(dtype)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    b, hk, hq, d, td = c["batch"], c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"], _dtype(c)
    n, lens = _counts(c), _lens(c)
    total, u, cap = sum(n), b * hk, max(lens) + max(n) + 1
    s = {"case": c, "counts": n}
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if c["kind"] != "rope" or c["cache"]:
        s["k"], s["v"] = _key_rows(g, (u, cap, d), td), _randn(g, (u, cap, d), td)
    if c["kind"] in ("rope", "verify"):
        s["qkv"] = _randn(g, (total, (hq + 2 * hk) * d), td)
        rot = c.get("rot", d)
        s["inv_freq"] = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float32,
                                     device="cuda")
        far = c.get("far", 0)
        first = torch.randint(0, far + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        base = torch.repeat_interleave(first + c["rows"], torch.tensor(n, device="cuda"), output_size=total)
        s["pos"] = base + torch.cat([torch.arange(x, dtype=torch.int32, device="cuda") for x in n])
        s["q_gain"] = 1.0 + 0.1 * _randn(g, (d,))
        s["k_gain"] = 1.0 + 0.1 * _randn(g, (d,))
        if c["kind"] == "rope" and not c["norm"]:
            s["q_gain"] = s["k_gain"] = None
    else:
        s["q"] = _randn(g, (total, hq, d), td)
    if c["kind"] in ("tree", "verify"):
        # node i hangs below one of the few nodes before it, as a drafter's best-first tree does
        t = torch.cat([torch.arange(x, device="cuda") for x in n])
        back = (torch.rand(total, generator=g, device="cuda") * 6).long() + 1
        s["parent"] = torch.clamp(t - back, min=-1).to(torch.int32)
    if c["kind"] == "verify":
        keep = _keeps(c)
        s["keep"] = torch.tensor(keep, dtype=torch.int32, device="cuda")
        wide = max(keep)
        # an accepted path: ascending nodes of each sequence (entries behind its count unused)
        path = [[min(x - 1, (i * x) // k) for i in range(wide)] for x, k in zip(n, keep)]
        s["path"] = torch.tensor(path, dtype=torch.int32, device="cuda")
        s["wide"] = wide
        s["next"] = c["rows"] + 7
        s["alpha"] = torch.rand((u, cap), generator=g, device="cuda")
        s["num"] = torch.rand((u, cap), generator=g, device="cuda", dtype=torch.float64)
        s["den"] = torch.rand((u, cap), generator=g, device="cuda", dtype=torch.float64)
        s["fpos"] = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(u, 1)
        s["vnorm"] = s["v"].float().square().sum(-1).sqrt()
        s["unit_len"] = s["lens"].clone()
    if own:
        _handles(c, s, cap, max(lens))
    return s


def _handles(c, s, cap, rows):
    """What a user's program keeps: the cache's buffers, the packed tokens, the rotation."""
    from paper_2608_08878_amd.buffers import DecodeBuffers, make_rope, make_tokens
    buf = DecodeBuffers(c["batch"], 1, c["kv_heads"] * c["group"], c["kv_heads"], c["head_dim"], cap, c["dtype"],
                        features=c["kind"] == "verify", ragged=c["uneven"] and c["kind"] in ("tree", "verify"))
    if "k" in s:
        buf.k.copy_(s["k"])
        buf.v.copy_(s["v"])
    if buf.unit_len is not None:
        buf.unit_len.copy_(s["lens"])
    buf.kv.len = rows
    if c["kind"] == "verify":
        for mine, theirs in ((buf.alpha, "alpha"), (buf.num, "num"), (buf.den, "den"), (buf.pos, "fpos"),
                             (buf.vnorm, "vnorm")):
            mine.copy_(s[theirs])
    s["buf"], s["tokens"] = buf, make_tokens(s["counts"])
    if "inv_freq" in s:
        s["rope"] = make_rope(s["inv_freq"], interleaved=c.get("interleaved", False), norm=c.get("norm", True), eps=EPS,
                              q_gain=s["q_gain"], k_gain=s["k_gain"])


def _projections(c, s):
    hk, hq, d = c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"]
    q, k, v = s["qkv"].split([hq * d, hk * d, hk * d], dim=1)
    return q.unflatten(1, (hq, d)), k.unflatten(1, (hk, d)), v.unflatten(1, (hk, d))


# ------------------------------------------------------------------------ plain forms

def _norm_rotate(x, gain, cos, sin, c):
    y = x.float()
    if c.get("norm", True):
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gain
    r = 2 * cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    if c.get("interleaved", False):
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _owners(s):
    """For every packed token its sequence and its number there."""
    t = torch.arange(s["counts_total"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu"], t, right=True) - 1
    return seq, (t - s["cu"][seq]).long()


def _plain_rope(c, s):
    q, k, v = _projections(c, s)
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _norm_rotate(q, s["q_gain"], cos, sin, c)
    k = _norm_rotate(k, s["k_gain"], cos, sin, c)
    if c["kind"] == "rope" and not c["cache"]:
        return q, k
    seq, r = _owners(s)
    unit = seq[:, None] * c["kv_heads"] + torch.arange(c["kv_heads"], device="cuda")
    slot = s["lens"].long()[unit] + r[:, None]
    s["k"][unit, slot] = k
    s["v"][unit, slot] = v
    return q, k


def _ancestors(parent, cu, n, most):
    """[batch][most][most]: whether node j is node i or above it."""
    b = n.shape[0]
    i = torch.arange(most, device="cuda")
    at = (cu[:-1, None] + i).clamp(max=parent.shape[0] - 1).long()
    p = torch.where(i < n[:, None], parent[at], -1)
    up = ((p[..., None] == i) & (p[..., None] < i[:, None])).double()
    eye = torch.eye(most, device="cuda", dtype=torch.float64).expand(b, -1, -1)
    return torch.linalg.matrix_power(eye + up, most) > 0


def _plain_attention(c, s, q):
    b, hk, grp, d = c["batch"], c["kv_heads"], c["group"], c["head_dim"]
    most, cu = max(s["counts"]), s["cu"]
    n = cu[1:] - cu[:-1]
    i = torch.arange(most, device="cuda")
    at = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1).long()
    qp = q[at].float().reshape(b, most, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * most, d)
    rows = s["k"].shape[1] - 1
    kf = s["k"][:, :rows].float().reshape(b, hk, rows, d)
    vf = s["v"][:, :rows].float().reshape(b, hk, rows, d)
    x = (torch.matmul(qp, kf.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(d))).reshape(b, hk, grp, most, rows)
    j = torch.arange(rows, device="cuda") - s["lens"].reshape(b, hk, 1)
    if c["kind"] == "prompt":
        sees = j[:, :, None] <= i[:, None]
    else:
        anc = _ancestors(s["parent"], cu, n, most)
        ext = torch.cat([anc, anc.new_ones(b, most, 1), anc.new_zeros(b, most, 1)], -1)
        at_j = torch.where(j < 0, most, torch.where(j < most, j, most + 1)).long()
        sees = ext[:, None].expand(b, hk, most, most + 2).gather(-1, at_j[:, :, None].expand(b, hk, most, rows))
    x.masked_fill_(~sees[:, :, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    o = torch.matmul(x.reshape(b, hk, grp * most, rows), vf) / x.sum(-1).reshape(b, hk, grp * most, 1)
    o = o.reshape(b, hk, grp, most, d).permute(0, 3, 1, 2, 4).reshape(b, most, hk * grp, d)
    seq, r = _owners(s)
    return o[seq, r].to(q.dtype)


def _plain_commit(c, s):
    b, hk = c["batch"], c["kv_heads"]
    u = torch.arange(b * hk, device="cuda")
    i = torch.arange(s["wide"], device="cuda")
    kept = (i < s["keep"][:, None]).repeat_interleave(hk, 0)
    start = s["lens"].long()[:, None]
    n = (s["cu"][1:] - s["cu"][:-1])[:, None]
    take = torch.minimum(torch.maximum(s["path"], i), n - 1).long().repeat_interleave(hk, 0)
    unit = u[:, None].expand_as(kept)[kept]
    src, dst = (start + take)[kept], (start + i)[kept]
    vr = s["v"][unit, src]
    s["k"][unit, dst] = s["k"][unit, src]
    s["v"][unit, dst] = vr
    s["alpha"][unit, dst] = 0
    s["num"][unit, dst] = 0
    s["den"][unit, dst] = 0
    s["fpos"][unit, dst] = (s["next"] + i).to(torch.int32).expand_as(kept)[kept]
    s["vnorm"][unit, dst] = vr.float().square().sum(-1).sqrt()
    s["unit_len"].copy_(s["lens"] + s["keep"].repeat_interleave(hk))


STATE = ("k", "v", "alpha", "num", "den", "fpos", "vnorm", "unit_len")


def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    s["counts_total"] = sum(s["counts"])
    if c["kind"] == "rope":
        q, k = _plain_rope(c, s)
        return [q, s["k"], s["v"]] if c["cache"] else [q, k]
    if c["kind"] != "verify":
        return [_plain_attention(c, s, s["q"])]
    q, _ = _plain_rope(c, s)
    o = _plain_attention(c, s, q)
    _plain_commit(c, s)
    return [o] + [s[x] for x in STATE]


def _run_own(c, s):
    buf = s["buf"]
    if c["kind"] == "rope":
        q, k, v = _projections(c, s)
        if c["cache"]:
            q, _ = buf.norm_rope(s["tokens"], s["rope"], q, k, v, s["pos"])
            return [q, buf.k, buf.v]
        return list(buf.norm_rope(s["tokens"], s["rope"], q, k, None, s["pos"]))
    if c["kind"] == "prompt":
        return [buf.prompt_attention(s["tokens"], s["q"])]
    if c["kind"] == "tree":
        return [buf.tree_attention(s["tokens"], s["parent"], s["q"])]
    # a speculative step from the same cache: its lengths as they were before the last pass
    buf.kv.len, buf.feat.next_pos = max(_lens(c)), s["next"]
    if buf.unit_len is not None:
        buf.unit_len.copy_(s["lens"])
    q, k, v = _projections(c, s)
    q, _ = buf.norm_rope(s["tokens"], s["rope"], q, k, v, s["pos"])
    o = buf.tree_attention(s["tokens"], s["parent"], q)
    if buf.unit_len is not None:
        buf.commit_rows(s["tokens"], s["path"], s["keep"])
        lens = buf.unit_len
    else:
        buf.commit_rows(s["tokens"], s["path"])
        lens = torch.full_like(s["lens"], buf.kv.len)
    return [o, buf.k, buf.v, buf.alpha, buf.num, buf.den, buf.pos, buf.vnorm, lens]


# ------------------------------------------------------------------------ 64 bits

def _exact_rope(c, s):
    hk, hq, d = c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"]
    x = s["qkv"].double().reshape(-1, hq + 2 * hk, d)
    parts = {"q": x[:, :hq].clone(), "k": x[:, hq:hq + hk].clone(), "v": x[:, hq + hk:]}
    half = s["inv_freq"].numel()
    phi = torch.outer(s["pos"].double(), s["inv_freq"].double())[:, None]
    z = torch.polar(torch.ones_like(phi), phi)
    if c.get("interleaved", False):
        first, second = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
    else:
        first, second = slice(0, half), slice(half, 2 * half)
    for name in ("q", "k"):
        y = parts[name]
        if c.get("norm", True):
            y /= ((y * y).sum(-1, keepdim=True) / d + EPS).sqrt()
            y *= s[name + "_gain"].double()
        w = torch.complex(y[..., first], y[..., second]) * z
        y[..., first], y[..., second] = w.real, w.imag
    return parts["q"], parts["k"], parts["v"]


def _exact_attention(c, s, q, k, v):
    hk, grp, d = c["kv_heads"], c["group"], c["head_dim"]
    out = torch.empty_like(q)
    lens, at = s["lens"].tolist(), 0
    parents = s["parent"].tolist() if "parent" in s else None
    for b, n in enumerate(s["counts"]):
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        if parents is not None:
            rows = []
            for i in range(n):
                p = parents[at + i]
                rows.append([i == j or (0 <= p < i and rows[p][j]) for j in range(n)])
            seen = torch.tensor(rows, device="cuda")
        for g in range(hk):
            u, r = b * hk + g, lens[b * hk + g]
            kk, vv = k[u, :r + n].double(), v[u, :r + n].double()
            for h in range(g * grp, (g + 1) * grp):
                w = q[at:at + n, h] @ kk.T / math.sqrt(d)
                w[:, r:][~seen] = -math.inf
                w = torch.exp(w - w.max(1, keepdim=True).values)
                out[at:at + n, h] = (w @ vv) / w.sum(1, keepdim=True)
        at += n
    return out


def exact(c, seed):
    s = prepare(c, seed)
    lens, hk = s["lens"].tolist(), c["kv_heads"]
    if c["kind"] in ("prompt", "tree"):
        return [_exact_attention(c, s, s["q"].double(), s["k"], s["v"])]
    q, k, v = _exact_rope(c, s)
    if c["kind"] == "rope" and not c["cache"]:
        return [q, k]
    ke, ve = s["k"].double(), s["v"].double()
    at = 0
    for b, n in enumerate(s["counts"]):
        for g in range(hk):
            u = b * hk + g
            ke[u, lens[u]:lens[u] + n] = k[at:at + n, g]
            ve[u, lens[u]:lens[u] + n] = v[at:at + n, g]
        at += n
    if c["kind"] == "rope":
        return [q, ke, ve]
    o = _exact_attention(c, s, q, ke, ve)
    alpha, num, den = s["alpha"].double(), s["num"].clone(), s["den"].clone()
    vnorm, fpos = s["v"].double().square().sum(-1).sqrt(), s["fpos"].clone()
    path, keep, ulen = s["path"].tolist(), s["keep"].tolist(), s["unit_len"].clone()
    for u, r in enumerate(lens):
        b = u // hk
        for j in range(keep[b]):
            t = min(max(path[b][j], j), s["counts"][b] - 1)
            ke[u, r + j], ve[u, r + j] = ke[u, r + t].clone(), ve[u, r + t].clone()
            alpha[u, r + j] = num[u, r + j] = den[u, r + j] = 0
            fpos[u, r + j] = s["next"] + j
            vnorm[u, r + j] = ve[u, r + j].square().sum().sqrt()
        ulen[u] = r + keep[b]
    return [o, ke, ve, alpha, num, den, fpos, vnorm, ulen]
