"""The operators for caches that are long or shared: the attention of sequences that have rows in
common (the rollouts of one prompt), the bounds of the keys of a cache's blocks, the choice of
blocks by those bounds, and the attention over chosen blocks.

With ``own`` false every operator is computed in its plain form (elementary torch operations in
float32, block scores in float64), with ``own`` true through the framework's entry points.
``exact`` is the same mathematics in float64, unit by unit.

Layouts: packed tokens of sequence b are cu[b] .. cu[b + 1] - 1; caches are [units][capacity][D],
unit b * Hk + g of sequence (or prefix) b and KV head g.  Token r of a sequence is row len + r of its
units.  A block is S successive rows; bounds are [units][capacity / S][2][D], the largest and the
smallest element of a block's keys; lists of blocks are [batch][groups][Hk][count], ascending with -1
behind, a group being `share` successive tokens of a sequence.
"""
import math

import torch

own = False


def _case(name, kind, **kw):
    c = {"name": name, "kind": kind, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16", "rows": 0,
         "tokens": 1, "uneven": False}
    c.update(kw)
    return c


def _shared(name, **kw):
    return _case(name, "shared", **{"prefixes": 1, "members": 8, "loose": 0, "tree": False, **kw})


def _blocks(name, kind, **kw):
    return _case(name, kind, **{"batch": 1, "block": 64, "count": 64, "share": 1, "first": 1, "last": 2, **kw})


def listed():
    return [
        # a step of four rollouts of the toy model's prompt in float32: latency
        _shared("shared_f32_toy", members=4, kv_heads=2, group=2, head_dim=64, dtype="f32", shared=512, rows=9),
        # the teacher's step of eight rollouts of one 8k prompt, each with a few hundred rows of its own
        _shared("shared_step_8k", shared=8192, rows=511, uneven=True),
        # four prompts of up to 16k rows, up to sixteen rollouts each, and three sequences without one
        _shared("shared_step_b59", prefixes=4, members=16, loose=3, shared=16384, rows=1024, uneven=True),
        # trees of up to 9 drafted tokens of sixteen rollouts, 64-element heads, eight queries to a key head
        _shared("shared_draft_d64", members=16, group=8, head_dim=64, shared=6001, rows=200, tokens=9, uneven=True,
                tree=True),
        # eight questions of 512 tokens about one text of 16k: the largest
        _shared("shared_prompts_16k", shared=16384, tokens=512),
        # the blocks of 16 prompts of 16k rows, after their prefill
        _blocks("bounds_16k_b16", "bounds", batch=16, rows=16384, start=0),
        # the blocks that the last 700 rows of the toy model's three caches touch
        _blocks("bounds_f32_next", "bounds", batch=3, kv_heads=2, group=2, head_dim=64, dtype="f32", rows=2049,
                start=1349, block=16, uneven=True),
        # a decode step of 16 sequences picks 64 of up to 512 blocks
        _blocks("select_step_b16", "select", batch=16, rows=32768, uneven=True),
        # parts of four prompts, 16 successive tokens picking 48 of 256 blocks of 32 rows together
        _blocks("select_part_8k", "select", batch=4, rows=8200, tokens=513, block=32, count=48, share=16, uneven=True),
        # the attention of that decode step: 4096 of up to 32768 rows
        _blocks("blocks_step_b16", "blocks", batch=16, rows=32768, uneven=True),
        # the next 512 tokens of one prompt over 64 of 512 blocks, 32 tokens together
        _blocks("blocks_part_32k", "blocks", rows=32768, tokens=512, share=32),
        # a whole step of one sequence with 100k rows: choice and attention, latency
        _blocks("sparse_step_100k", "sparse", rows=100001, count=48),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "shared", "shared", "bounds", "select", "select", "blocks", "blocks",
                       "sparse"])
    c = {"kind": kind, "kv_heads": rng.choice([1, 2, 4, 8, 8]), "group": rng.choice([1, 2, 4, 4, 8]),
         "head_dim": rng.choice([64, 128, 128]), "dtype": "f32" if rng.random() < 0.15 else "bf16",
         "uneven": rng.random() < 0.6}
    fewer = 4 if c["dtype"] == "f32" else 1
    if kind == "shared":
        c.update(prefixes=_log(rng, 1, 6), members=_log(rng, 1, 24), loose=rng.choice([0, 0, 1, 4]),
                 shared=_log(rng, 8, 16384), rows=_log(rng, 1, 1024) - 1, tree=rng.random() < 0.3)
        c["tokens"] = 1 if rng.random() < 0.5 else _log(rng, 1, 64 if c["tree"] else 512)
        while c["tokens"] > 1 and work({**c, "name": ""})["flops"] > 1.1e12 / fewer:
            c["tokens"] //= 2
        return c
    c.update(batch=_log(rng, 1, 16), block=rng.choice([16, 32, 64, 64, 128]), count=_log(rng, 3, 64), share=1,
             first=rng.choice([0, 1]), last=rng.choice([0, 1, 2]), rows=_log(rng, 20, 100001), tokens=1)
    c["rows"] = max(c["block"], min(c["rows"], 4194304 // (c["batch"] * c["kv_heads"] * fewer)))
    if kind == "bounds":
        c["start"] = 0 if rng.random() < 0.6 else rng.randrange(c["rows"])
    elif rng.random() < 0.4:
        c["tokens"], c["share"] = _log(rng, 1, 512), rng.choice([1, 4, 16, 32, 50])
        c["batch"] = max(1, min(c["batch"], 1024 // c["tokens"]))
        if c["share"] < 16:
            c["tokens"] = min(c["tokens"], 64)
    return c


# ------------------------------------------------------------------------ sizes

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _members(c):
    """Sequences of every prefix: `members`, or the first that many and the others fewer."""
    m = c["members"]
    return [m - (m * ((3 * p) % 5)) // 7 if c["uneven"] else m for p in range(c["prefixes"])]


def _batch(c):
    return sum(_members(c)) + c["loose"] if c["kind"] == "shared" else c["batch"]


def _counts(c):
    """Tokens of each sequence."""
    n = c["tokens"]
    if not c["uneven"]:
        return [n] * _batch(c)
    return [max(1, n - (n * ((5 * b) % 8)) // 9) for b in range(_batch(c))]


def _fewer(most, units, uneven):
    return [max(0, most - (most * ((3 * i) % 7)) // 13) if uneven else most for i in range(units)]


def _lens(c):
    """Rows of each unit before the call."""
    return _fewer(c["rows"], _batch(c) * c["kv_heads"], c["uneven"])


def _shared_lens(c):
    return _fewer(c["shared"], c["prefixes"] * c["kv_heads"], c["uneven"])


def _groups(c):
    return -(-c["tokens"] // c["share"])


def work(c):
    n, hk, grp, d = _counts(c), c["kv_heads"], c["group"], c["head_dim"]
    e, lens = (4 if c["dtype"] == "f32" else 2), _lens(c)
    ends = 2 * sum(n) * hk * grp * d * e                     # queries and outputs
    if c["kind"] == "shared":
        sl, pairs, b = _shared_lens(c), 0, 0
        for p, m in enumerate(_members(c) + [c["loose"]]):
            for x in n[b:b + m]:
                own_rows = sum(lens[b * hk:(b + 1) * hk])
                pairs += x * (own_rows + (sum(sl[p * hk:(p + 1) * hk]) if p < c["prefixes"] else 0))
                pairs += hk * x * (x + 1) // 2
                b += 1
        rows = sum(sl) + sum(lens) + hk * sum(n)
        return {"bytes": ends + 2 * rows * d * e, "flops": 4 * d * grp * pairs}
    S = c["block"]
    if c["kind"] == "bounds":
        blocks = sum(max(0, x // S - c["start"] // S) for x in lens)
        return {"bytes": blocks * (S + 2) * d * e, "flops": 2 * blocks * S * d}
    cand = [x // S for x in lens]
    lists = [-(-x // c["share"]) for x in n]
    choice = {"bytes": sum(n) * hk * grp * d * e + 2 * d * e * sum(cand) + 4 * sum(lists) * hk * c["count"],
              "flops": sum(4 * d * lists[u // hk] * x for u, x in enumerate(cand))}
    if c["kind"] == "select":
        return choice
    rows = pairs = 0
    for u, x in enumerate(cand):
        b, k = u // hk, min(c["count"], x)
        seen = x * (1 - (1 - k / x) ** lists[b]) if x else 0        # blocks that one of the lists holds
        rows += seen * S + lens[u] - x * S + n[b]
        pairs += grp * n[b] * (k * S + lens[u] - x * S + (n[b] + 1) / 2)
    att = {"bytes": int(ends + 2 * rows * d * e), "flops": int(4 * d * pairs)}
    if c["kind"] == "blocks":
        return att
    return {"bytes": choice["bytes"] + att["bytes"], "flops": choice["flops"] + att["flops"]}


# ------------------------------------------------------------------------ inputs

def _randn(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _key_rows(g, u, cap, d, dtype):
    """Keys with log-normal norms around a center that lies off zero, by channel, and moves along the rows."""
    x = torch.randn((u, cap, d), generator=g, device="cuda")
    x *= torch.exp(0.4 * torch.randn((u, cap, 1), generator=g, device="cuda"))
    x += 0.5 * _randn(g, (u, 1, d))
    x += 0.6 * _randn(g, (u, -(-cap // 50), d)).repeat_interleave(50, 1)[:, :cap]
    return x.to(dtype)


def _offsets(counts):
    cu = [0]
    for x in counts:
        cu.append(cu[-1] + x)
    return cu


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    hk, hq, d, td = c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"], _dtype(c)
    n, lens, u = _counts(c), _lens(c), _batch(c) * c["kv_heads"]
    cap = c["rows"] + c["tokens"] + 3
    s = {"case": c, "counts": n, "total": sum(n)}
    s["cu"] = torch.tensor(_offsets(n), dtype=torch.int32, device="cuda")
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["k"] = _key_rows(g, u, cap, d, td)
    if c["kind"] != "bounds":
        s["q"] = _randn(g, (sum(n), hq, d), td)
    if c["kind"] in ("shared", "blocks", "sparse"):
        s["v"] = _randn(g, (u, cap, d), td)
    if c["kind"] == "shared":
        up = c["prefixes"] * hk
        s["pk"] = _key_rows(g, up, c["shared"] + 1, d, td)
        s["pv"] = _randn(g, (up, c["shared"] + 1, d), td)
        s["plens"] = torch.tensor(_shared_lens(c), dtype=torch.int32, device="cuda")
        if c["tree"]:
            # node i hangs below one of the few nodes before it, as a drafter's best-first tree does
            t = torch.cat([torch.arange(x, device="cuda") for x in n])
            back = (torch.rand(sum(n), generator=g, device="cuda") * 6).long() + 1
            s["parent"] = torch.clamp(t - back, min=-1).to(torch.int32)
    else:
        s["bounds"] = torch.zeros((u, cap // c["block"], 2, d), dtype=td, device="cuda")
    if c["kind"] in ("select", "sparse"):
        _plain_bounds(c, s, 0)
    if c["kind"] == "blocks":
        # a random choice of every group, in ascending order
        cand = (s["lens"] // c["block"]).view(c["batch"], 1, hk, 1).clamp(min=0)
        most = max(c["count"], c["rows"] // c["block"])
        x = torch.rand((c["batch"], _groups(c), hk, most), generator=g, device="cuda")
        i = torch.arange(most, device="cuda")
        x = torch.where(i < cand, x, -1.0)
        val, at = x.topk(c["count"], -1)
        at = torch.where(val >= 0, at, most).sort(-1).values
        at = torch.where(at < most, at, -1)
        live = torch.arange(_groups(c), device="cuda") * c["share"] < (s["cu"][1:] - s["cu"][:-1])[:, None]
        s["list"] = torch.where(live[:, :, None, None], at, -1).to(torch.int32).contiguous()
    if own:
        _handles(c, s, cap)
    return s


def _buffers(c, batch, cap, k, v, lens, rows):
    from paper_2608_08878_amd.buffers import DecodeBuffers
    buf = DecodeBuffers(batch, 1, c["kv_heads"] * c["group"], c["kv_heads"], c["head_dim"], cap, c["dtype"],
                        features=False, ragged=c["uneven"])
    buf.k.copy_(k)
    if v is not None:
        buf.v.copy_(v)
    if buf.unit_len is not None:
        buf.unit_len.copy_(lens)
    buf.kv.len = rows
    return buf


def _handles(c, s, cap):
    """What a user's program keeps: the cache's buffers, the packed tokens, the prefixes or blocks."""
    from paper_2608_08878_amd.buffers import make_shared, make_tokens
    buf = s["buf"] = _buffers(c, _batch(c), cap, s["k"], s.get("v"), s["lens"], c["rows"])
    s["tokens"] = make_tokens(s["counts"])
    if c["kind"] == "shared":
        pre = _buffers(c, c["prefixes"], c["shared"] + 1, s["pk"], s["pv"], s["plens"], c["shared"])
        s["shared"] = make_shared(pre, _members(c))
    else:
        s["blocks"] = buf.make_blocks(c["block"])
        s["blocks"].bounds_tensor.copy_(s["bounds"])


# ------------------------------------------------------------------------ plain forms

def _padded(s, b, most):
    """For every sequence its tokens' places in the packed arrays, `most` of them."""
    i = torch.arange(most, device="cuda")
    return (s["cu"][:-1, None] + i).clamp(max=s["total"] - 1).long()


def _owners(s):
    """For every packed token its sequence and its number there."""
    t = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu"], t, right=True) - 1
    return seq, (t - s["cu"][seq]).long()


def _ancestors(parent, cu, n, most):
    """[batch][most][most]: whether node j is node i or above it."""
    i = torch.arange(most, device="cuda")
    at = (cu[:-1, None] + i).clamp(max=parent.shape[0] - 1).long()
    p = torch.where(i < n[:, None], parent[at], -1)
    up = ((p[..., None] == i) & (p[..., None] < i[:, None])).double()
    eye = torch.eye(most, device="cuda", dtype=torch.float64).expand(n.shape[0], -1, -1)
    return torch.linalg.matrix_power(eye + up, most) > 0


def _plain_shared(c, s):
    b, hk, grp, d = _batch(c), c["kv_heads"], c["group"], c["head_dim"]
    most, cu, cap = max(s["counts"]), s["cu"], s["k"].shape[1]
    n = cu[1:] - cu[:-1]
    i = torch.arange(most, device="cuda")
    q = s["q"][_padded(s, b, most)].float().reshape(b, most, hk, grp, d).permute(0, 2, 3, 1, 4)
    q = (q * (1.0 / math.sqrt(d))).reshape(b, hk, grp * most, d)
    kf, vf = s["k"].float().reshape(b, hk, cap, d), s["v"].float().reshape(b, hk, cap, d)
    x = torch.matmul(q, kf.transpose(-1, -2).contiguous()).reshape(b, hk, grp, most, cap)
    j = torch.arange(cap, device="cuda") - s["lens"].reshape(b, hk, 1)
    if not c["tree"]:
        sees = j[:, :, None] <= i[:, None]
    else:
        anc = _ancestors(s["parent"], cu, n, most)
        ext = torch.cat([anc, anc.new_ones(b, most, 1), anc.new_zeros(b, most, 1)], -1)
        at_j = torch.where(j < 0, most, torch.where(j < most, j, most + 1)).long()
        sees = ext[:, None].expand(b, hk, most, most + 2).gather(-1, at_j[:, :, None].expand(b, hk, most, cap))
    x = x.masked_fill_(~sees[:, :, None], -math.inf).reshape(b, hk, grp * most, cap)
    out = torch.empty((b, hk, grp * most, d), device="cuda")
    b0 = 0
    for p, m in enumerate(_members(c) + [c["loose"]]):
        if m == 0:
            continue
        own_x, part = x[b0:b0 + m], slice(b0, b0 + m)
        top = own_x.amax(-1, keepdim=True)
        if p < c["prefixes"]:
            pk, pv = s["pk"][p * hk:(p + 1) * hk].float(), s["pv"][p * hk:(p + 1) * hk].float()
            qp = q[part].transpose(0, 1).reshape(hk, m * grp * most, d)
            y = torch.matmul(qp, pk.transpose(-1, -2).contiguous())
            gone = torch.arange(pk.shape[1], device="cuda") >= s["plens"][p * hk:(p + 1) * hk, None]
            y.masked_fill_(gone[:, None], -math.inf)
            y = y.reshape(hk, m, grp * most, -1).transpose(0, 1)
            top = torch.maximum(top, y.amax(-1, keepdim=True))
            y = (y - top).exp_()
            own_x = (own_x - top).exp_()
            o = torch.matmul(y.transpose(0, 1).reshape(hk, m * grp * most, -1), pv)
            o = o.reshape(hk, m, grp * most, d).transpose(0, 1) + torch.matmul(own_x, vf[part])
            out[part] = o / (y.sum(-1, keepdim=True) + own_x.sum(-1, keepdim=True))
        else:
            own_x = (own_x - top).exp_()
            out[part] = torch.matmul(own_x, vf[part]) / own_x.sum(-1, keepdim=True)
        b0 += m
    out = out.reshape(b, hk, grp, most, d).permute(0, 3, 1, 2, 4).reshape(b, most, hk * grp, d)
    seq, r = _owners(s)
    return out[seq, r].to(s["q"].dtype)


def _plain_bounds(c, s, start):
    S, k = c["block"], s["k"]
    u, cap, d = k.shape
    whole = k[:, :cap // S * S].reshape(u, cap // S, S, d)
    new = torch.stack([whole.amax(2), whole.amin(2)], 2)
    j = torch.arange(cap // S, device="cuda")
    due = (j >= start // S) & (j < (s["lens"] // S)[:, None])
    s["bounds"].copy_(torch.where(due[:, :, None, None], new, s["bounds"]))
    return s["bounds"]


def _plain_select(c, s):
    b, hk, grp, d, S = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["block"]
    most, share, groups = max(s["counts"]), c["share"], _groups(c)
    n = s["cu"][1:] - s["cu"][:-1]
    q = s["q"][_padded(s, b, groups * share)].double()
    q = q * (torch.arange(groups * share, device="cuda") < n[:, None])[..., None, None]
    q = q.reshape(b, groups, share, hk, grp, d)
    up, down = q.clamp(min=0).sum((2, 4)).transpose(1, 2), q.clamp(max=0).sum((2, 4)).transpose(1, 2)
    nb = s["bounds"].shape[1]
    bd = s["bounds"].double().reshape(b, hk, nb, 2 * d)
    x = torch.matmul(torch.cat([up, down], -1), bd.transpose(-1, -2).contiguous()).transpose(1, 2)
    cand = (s["lens"] // S).view(b, 1, hk, 1)
    j = torch.arange(nb, device="cuda")
    x = torch.where((j < c["first"]) | (j >= cand - c["last"]), math.inf, x)
    x = torch.where(j < cand, x, -math.inf)
    live = torch.arange(groups, device="cuda") * share < n[:, None]
    if nb < c["count"]:
        x = torch.nn.functional.pad(x, (0, c["count"] - nb), value=-math.inf)
    x, at = x.sort(dim=-1, descending=True, stable=True)
    k = torch.arange(c["count"], device="cuda")
    at = torch.where(k < cand, at[..., :c["count"]], 1 << 30).sort(-1).values
    at = torch.where(at < 1 << 30, at, -1)
    return torch.where(live[:, :, None, None], at, -1).to(torch.int32)


def _plain_blocks(c, s, chosen):
    b, hk, grp, d, S = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["block"]
    share, groups, cap = c["share"], _groups(c), s["k"].shape[1]
    cand = (s["lens"] // S).view(b, 1, hk, 1).long()
    rows = (chosen.long()[..., None] * S + torch.arange(S, device="cuda")).flatten(-2)
    ok = (chosen >= 0).repeat_interleave(S, -1)
    tail = cand * S + torch.arange(S - 1 + c["tokens"], device="cuda")
    rows = torch.cat([rows, tail.expand(b, groups, hk, -1)], -1).clamp(0, cap - 1)
    unit = (torch.arange(b, device="cuda")[:, None] * hk + torch.arange(hk, device="cuda")).view(b, 1, hk, 1)
    kf, vf = s["k"][unit, rows].float(), s["v"][unit, rows].float()
    q = s["q"][_padded(s, b, groups * share)].float().reshape(b, groups, share, hk, grp, d)
    q = q.permute(0, 1, 3, 2, 4, 5).reshape(b, groups, hk, share * grp, d) * (1.0 / math.sqrt(d))
    x = torch.matmul(q, kf.transpose(-1, -2).contiguous())
    r = torch.arange(groups * share, device="cuda").view(1, groups, 1, share, 1)
    end = s["lens"].view(b, 1, hk, 1, 1) + r + 1                    # rows that a token sees end here
    sees = torch.cat([ok[..., None, :].expand(-1, -1, -1, share, -1), tail[..., None, :] < end], -1)
    x.masked_fill_(~sees.repeat_interleave(grp, 3), -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    o = torch.matmul(x, vf) / x.sum(-1, keepdim=True)
    o = o.reshape(b, groups, hk, share, grp, d).permute(0, 1, 3, 2, 4, 5).reshape(b, groups * share, hk * grp, d)
    seq, at = _owners(s)
    return o[seq, at].to(s["q"].dtype)


def run(s):
    c = s["case"]
    if own:
        return _run_own(c, s)
    if c["kind"] == "shared":
        return [_plain_shared(c, s)]
    if c["kind"] == "bounds":
        return [_plain_bounds(c, s, c["start"])]
    if c["kind"] == "select":
        return [_plain_select(c, s)]
    if c["kind"] == "blocks":
        return [_plain_blocks(c, s, s["list"])]
    chosen = _plain_select(c, s)
    return [chosen, _plain_blocks(c, s, chosen)]


def _run_own(c, s):
    buf = s["buf"]
    if c["kind"] == "shared":
        return [buf.shared_attention(s["tokens"], s["shared"], s["q"], s.get("parent"))]
    if c["kind"] == "bounds":
        buf.block_bounds(s["blocks"], c["start"])
        return [s["blocks"].bounds_tensor]
    pick = {"count": c["count"], "share": c["share"], "first": c["first"], "last": c["last"]}
    if c["kind"] == "select":
        return [buf.block_select(s["tokens"], s["blocks"], s["q"], **pick)]
    if c["kind"] == "blocks":
        return [buf.block_attention(s["tokens"], s["blocks"], s["list"], s["q"], share=c["share"])]
    chosen = buf.block_select(s["tokens"], s["blocks"], s["q"], **pick)
    return [chosen, buf.block_attention(s["tokens"], s["blocks"], chosen, s["q"], share=c["share"])]


# ------------------------------------------------------------------------ 64 bits

def _attend(q, k, v, sees):
    """q [rows][D], k, v [keys][D], sees [rows][keys], float64."""
    w = q @ k.T / math.sqrt(q.shape[1])
    w[~sees] = -math.inf
    w = torch.exp(w - w.max(1, keepdim=True).values)
    return (w @ v) / w.sum(1, keepdim=True)


def _exact_shared(c, s):
    hk, grp = c["kv_heads"], c["group"]
    lens, plens = s["lens"].tolist(), s["plens"].tolist()
    parents = s["parent"].tolist() if c["tree"] else None
    q, out, at, b = s["q"].double(), torch.empty_like(s["q"], dtype=torch.float64), 0, 0
    for p, m in enumerate(_members(c) + [c["loose"]]):
        for b in range(b, b + m):
            n = s["counts"][b]
            seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
            if parents is not None:
                rows = []
                for i in range(n):
                    up = parents[at + i]
                    rows.append([i == j or (0 <= up < i and rows[up][j]) for j in range(n)])
                seen = torch.tensor(rows, device="cuda")
            for g in range(hk):
                u, L = b * hk + g, lens[b * hk + g]
                kk, vv = s["k"][u, :L + n].double(), s["v"][u, :L + n].double()
                before = L
                if p < c["prefixes"]:
                    before += plens[p * hk + g]
                    kk = torch.cat([s["pk"][p * hk + g, :plens[p * hk + g]].double(), kk])
                    vv = torch.cat([s["pv"][p * hk + g, :plens[p * hk + g]].double(), vv])
                sees = torch.cat([seen.new_ones(n, before), seen], 1)
                for h in range(g * grp, (g + 1) * grp):
                    out[at:at + n, h] = _attend(q[at:at + n, h], kk, vv, sees)
            at += n
        b += m > 0
    return out


def _exact_bounds(c, s):
    out, S = s["bounds"].double(), c["block"]
    for u, L in enumerate(s["lens"].tolist()):
        j0, j1 = c["start"] // S, L // S
        if j1 > j0:
            rows = s["k"][u, j0 * S:j1 * S].double().view(j1 - j0, S, -1)
            out[u, j0:j1, 0], out[u, j0:j1, 1] = rows.max(1).values, rows.min(1).values
    return out


def _exact_select(c, s):
    hk, grp, S, share = c["kv_heads"], c["group"], c["block"], c["share"]
    out = torch.full((c["batch"], _groups(c), hk, c["count"]), -1, dtype=torch.int32)
    lens, at = s["lens"].tolist(), 0
    q, bounds = s["q"].double(), s["bounds"].double()
    for b, n in enumerate(s["counts"]):
        for g in range(hk):
            nc = lens[b * hk + g] // S
            hi, lo = bounds[b * hk + g, :nc, 0], bounds[b * hk + g, :nc, 1]
            for i in range(-(-n // share)):
                x = q[at + i * share:at + min((i + 1) * share, n), g * grp:(g + 1) * grp].reshape(-1, q.shape[-1])
                score = (x.clamp(min=0) @ hi.T + x.clamp(max=0) @ lo.T).sum(0).tolist()
                # the first and last blocks, then the others by score
                held = [j for j in range(nc) if j < c["first"] or j >= nc - c["last"]]
                rest = sorted(set(range(nc)) - set(held), key=lambda j: (-score[j], j))
                pick = sorted((held + rest)[:c["count"]])
                out[b, i, g, :len(pick)] = torch.tensor(pick, dtype=torch.int32)
        at += n
    return out.cuda()


def _exact_blocks(c, s, chosen):
    hk, grp, S, share = c["kv_heads"], c["group"], c["block"], c["share"]
    q, out, at = s["q"].double(), torch.empty_like(s["q"], dtype=torch.float64), 0
    lens, chosen = s["lens"].tolist(), chosen.cpu()
    for b, n in enumerate(s["counts"]):
        for g in range(hk):
            u, L = b * hk + g, lens[b * hk + g]
            for i in range(-(-n // share)):
                t0, t1 = i * share, min((i + 1) * share, n)
                rows = [torch.arange(j * S, (j + 1) * S) for j in chosen[b, i, g].tolist() if j >= 0]
                old = sum(map(len, rows)) + L % S
                rows = torch.cat(rows + [torch.arange(L // S * S, L + t1)]).cuda()
                kk, vv = s["k"][u, rows].double(), s["v"][u, rows].double()
                r = torch.arange(t0, t1, device="cuda")[:, None]
                sees = torch.arange(len(rows), device="cuda") - old <= r
                for h in range(g * grp, (g + 1) * grp):
                    out[at + t0:at + t1, h] = _attend(q[at + t0:at + t1, h], kk, vv, sees)
        at += n
    return out


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "shared":
        return [_exact_shared(c, s)]
    if c["kind"] == "bounds":
        return [_exact_bounds(c, s)]
    if c["kind"] == "blocks":
        return [_exact_blocks(c, s, s["list"])]
    chosen = _exact_select(c, s)
    return [chosen] if c["kind"] == "select" else [chosen, _exact_blocks(c, s, chosen)]
