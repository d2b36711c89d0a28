"""Several tokens at once on the GPU: what a cache and its buffers keep from call to call."""
import numpy as np
import pytest
import torch

from oracle import prompt as op
from oracle import select as osel
from oracle import unit as ounit
from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers, make_policy, make_rope, make_tokens

from . import harness as H
from .test_gpu_prompt import MANY, Cache, check_attention, close, random_tree, uneven

pytestmark = pytest.mark.gpu


def test_a_captured_attention_keeps_its_workspace():
    # outgrown after the capture, with memory of its size taken by others since
    c = Cache([9], 3000, "bf16", 128, 2, 4, seed=50)
    want = c.buf.prompt_attention(c.tokens, c.q)
    assert c.buf.ws_bytes > 0
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.buf.prompt_attention(c.tokens, c.q, out=out)
    size = c.buf.ws_bytes
    c.buf.reserve_workspace(200000)
    assert c.buf.ws_bytes > size
    taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all((x == 255).all() for x in taken)
        assert torch.equal(c.buf.prompt_attention(c.tokens, c.q), want)     # eager, in the present one


def test_short_paths_fill_a_cache_to_its_capacity():
    # 8 drafted tokens a step, of which one or two stay: more steps than the capacity holds drafts
    c = Cache([8, 8], 20, "bf16", 64, 1, 2, seed=51, spare=40, lens=[20, 20])        # capacity 68
    buf, path = c.buf, torch.tensor([[1, 4], [0, 3]], dtype=torch.int32, device="cuda")
    keep = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    chain = torch.arange(-1, 7, dtype=torch.int32, device="cuda").repeat(2)
    lens = [20, 20]
    for step in range(20):
        new = buf.k[torch.arange(2), torch.tensor([n + p for n, p in zip(lens, (1, 0))])].clone()
        c.lens = lens
        check_attention(c, buf.tree_attention(c.tokens, chain, c.q), 0, [op.causal_mask(8)] * 2)
        buf.commit_rows(c.tokens, path, keep)
        assert buf.tighten_len() == lens[0] + 2 == buf.unit_len.max()
        assert torch.equal(buf.k[torch.arange(2), torch.tensor(lens)], new)
        lens = [lens[0] + 2, lens[1] + 1]
    assert buf.unit_len.tolist() == lens == [60, 40]
    with pytest.raises(B.DCError):                      # 60 rows and 8 tokens are the capacity's 68
        buf.commit_rows(make_tokens([9, 9]), width=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("counts,rows,hk", [([130] * 12, 300, 8), ([60] * 40, 300, 8), ([3], 300, 1), ([8] * 64, 300, 8)])
def test_values_near_the_largest_number(dtype, tree, counts, rows, hk):
    # one key 7.5 powers of two above all others, its value 3e36: the output is finite, though 2^7.5 of it
    # leave float32's range
    c = Cache(counts, rows, dtype, 128, hk, 1, seed=70)
    c.q.fill_(1.0)
    c.buf.k.zero_()
    c.buf.k[:, 200] = 7.5 * np.log(2) * 128 ** 0.5 / 128
    c.buf.v[:, 200] = 3e36
    if tree:
        out = c.buf.tree_attention(c.tokens, torch.full((c.N,), -1, dtype=torch.int32, device="cuda"), c.q)
        masks = [op.tree_mask([-1] * n) for n in counts]
    else:
        out, masks = c.buf.prompt_attention(c.tokens, c.q), [op.causal_mask(n) for n in counts]
    assert torch.isfinite(out.float()).all()
    check_attention(c, out, 0, masks)


def test_padding_around_the_sequences_is_left():
    # two tokens before the first sequence and three behind the last
    c = Cache([5, 0, 9], 40, "bf16", 128, 2, 4, seed=71, lens=[40, 38, 40, 40, 7, 30])
    t = make_tokens([5, 0, 9])
    t.tokens = 19
    t.cu_tensor.copy_(torch.tensor([2, 7, 7, 16], dtype=torch.int32))
    wide = [torch.randn((19, h, 128), generator=c.g).to(c.td).cuda() for h in (8, 2, 2)]
    pos = torch.randint(0, 900, (19,), generator=c.g, dtype=torch.int32).cuda()
    rope = make_rope(torch.rand(64, generator=c.g).cuda(), norm=True)
    tight = [x[2:16].contiguous() for x in wide]
    want, _ = c.buf.norm_rope(c.tokens, rope, *tight, pos[2:16].contiguous())
    k, v = c.buf.k.clone(), c.buf.v.clone()
    for u, r in enumerate(c.lens):
        n = [5, 0, 9][u // 2]
        c.buf.k[u, r:r + n], c.buf.v[u, r:r + n] = 3, 4
    got, _ = c.buf.norm_rope(t, rope, *wide, pos)
    assert torch.equal(got[2:16], want) and torch.equal(c.buf.k, k) and torch.equal(c.buf.v, v)
    heads = [x.contiguous() for x in (got[:2], got[16:])]
    for x, at in zip(heads, (slice(0, 2), slice(16, 19))):          # the padding's heads are turned like any
        one = make_tokens([x.shape[0]])
        alone = DecodeBuffers(1, 1, 8, 2, 128, 8, "bf16", features=False)
        assert torch.equal(alone.norm_rope(one, rope, wide[0][at], wide[1][at], None, pos[at].contiguous())[0], x)
    parent = torch.full((19,), -1, dtype=torch.int32, device="cuda")
    for tree in (False, True):
        out = torch.full((19, 8, 128), 5.0, dtype=c.td, device="cuda")
        a = c.buf.tree_attention(t, parent, got, out=out) if tree else c.buf.prompt_attention(t, got, out=out)
        b = c.buf.tree_attention(c.tokens, parent[:14].contiguous(), want) if tree else \
            c.buf.prompt_attention(c.tokens, want)
        assert (a[:2] == 5).all() and (a[16:] == 5).all()
        assert close(a[2:16], b, 50, float(c.buf.v.abs().max()), "bf16")
    c.buf.commit_rows(t)
    assert c.buf.unit_len.tolist() == [45, 43, 40, 40, 16, 39]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("counts,rows,hk,G,lens", MANY)
def test_trees_of_many_rows_do_not_depend_on_other_branches(dtype, D, counts, rows, hk, G, lens):
    # every tile shape: a node's rows infinite or NaN, which reaches the nodes below it alone
    if max(counts) > 256:
        counts = [256, 17]
    print(f"branches {dtype} D={D} counts={counts[:4]}", flush=True)
    c = Cache(counts, rows, dtype, D, hk, G, 1, uneven(len(counts) * hk, rows) if lens else None, seed=rows + D)
    parents = [random_tree(n, 5 * b + n) for b, n in enumerate(counts)]
    flat = torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda")
    want = c.buf.tree_attention(c.tokens, flat, c.q)
    for b, _, n in c.spans():
        for h in range(hk if n else 0):
            u = c.unit(b, 0, h)
            at = c.lens[u] + n // 2
            c.buf.v[u, at] = float("inf") if h % 2 else float("nan")
            c.buf.k[u, at] = float("nan") if h % 2 else -float("inf")
    got = c.buf.tree_attention(c.tokens, flat, c.q)
    for b, t0, n in c.spans():
        if n == 0:
            continue
        sees = torch.from_numpy(op.tree_mask(parents[b])[:, n // 2].copy()).cuda()
        g, w = got[t0:t0 + n], want[t0:t0 + n]
        assert close(g[~sees], w[~sees], rows + max(counts), 6, dtype), b
        assert not torch.isfinite(g[sees].float()).any(), b


# ------------------------------------------- sequences that see different numbers of tokens

class Sequences:
    """A cache of a few of the sequences of a seeded batch, fed by hand: rows written behind the
    cache's, committed, decoded over, evicted.  A sequence's numbers do not depend on the others."""

    def __init__(self, which, hk, G, D, window, ragged, sigma, cap, seed=60):
        self.which, self.hk, self.G, self.D, self.seed = which, hk, G, D, seed
        self.buf = DecodeBuffers(len(which), 1, hk * G, hk, D, cap, "bf16", window, features=True, sigma=sigma,
                                 ragged=ragged)

    def lens(self):
        if self.buf.unit_len is not None:
            return self.buf.unit_len.tolist()
        return [self.buf.kv.len] * self.buf.U

    def draw(self, what, b, *shape):
        g = torch.Generator().manual_seed(1000 * self.seed + 100 * what + b)
        return torch.randn(shape, generator=g).to(torch.bfloat16).cuda()

    def rows(self, what, b, count):
        return self.draw(what, b, 2, self.hk, count, self.D)

    def commit(self, what, counts, path=None, keep=None):
        """counts[b] new rows in every unit of sequence b, of which the path's first keep[b] stay."""
        rows = [self.rows(what, b, n) for b, n in zip(self.which, counts)]
        for u, r in enumerate(self.lens()):
            b, h = divmod(u, self.hk)
            self.buf.k[u, r:r + counts[b]], self.buf.v[u, r:r + counts[b]] = rows[b][0, h], rows[b][1, h]
        dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.buf.commit_rows(make_tokens(counts), dev(path), dev(keep))

    def inputs(self, what):
        """q, k, v of one step."""
        q = torch.cat([self.draw(what, b, self.hk, self.G, self.D) for b in self.which])
        kv = torch.stack([self.draw(what + 1, b, 2, self.hk, self.D) for b in self.which], 1)
        return q, kv[0].flatten(0, 1), kv[1].flatten(0, 1)

    def state(self, b):
        """Of every unit of sequence b, its rows by position."""
        out = []
        lens = self.lens()
        for h in range(self.hk):
            u = self.which.index(b) * self.hk + h
            d = {n: H.to_np(getattr(self.buf, n)[u, :lens[u]]).astype(np.float64)
                 for n in ("k", "v", "pos", "alpha", "num", "den", "vnorm")}
            if self.buf.sigma is not None:
                d["sigma"] = H.to_np(self.buf.sigma[u, :lens[u]]).astype(np.float64)
            out.append(H.by_position(d))
        return out


PROMPT, KEEP = [40, 7, 0, 23, 31], [3, 1, 2, 0, 2]
PATH = [[0, 1, 3], [2, 3, 3], [0, 2, 3], [0, 1, 2], [1, 2, 3]]
# (hidden widths, inputs, LayerNorm): every scoring pass that reads pos / T
POLICIES = [((32,), 4, False), ((32,), 4, True), ((24,), 5, False), ((64, 64), 4, False), ((64, 48), 4, True)]


def _params(hidden, n_in, ln):
    g = torch.Generator().manual_seed(9)
    size, width = 0, n_in
    for h in hidden:
        size += h * width + h + (2 * h if ln else 0)
        width = h
    return (0.4 * torch.randn(size + width + 1, generator=g)).cuda()


def _same(a, b, names, at):
    for x, y in zip(a, b):
        assert len(x["pos"]) == len(y["pos"]) > 0
        assert np.array_equal(x["pos"], y["pos"]), (at, x["pos"], y["pos"])
        for n in names:
            ok, worst = H.vec_ok(x[n], y[n], tol=2 * H.FP_TOL)      # either side within the rule of one
            assert ok, (at, n, worst)


def _run(s, prompt, budget, pol, units, each):
    """The same steps on a batch or on one of its sequences; each(stage, scores or None) looks in between."""
    pick = lambda x: [x[b % 5] for b in s.which]  # noqa: E731
    alone = s.buf.unit_len is None
    counts = pick(prompt)
    if max(counts) > 0:
        s.commit(1, counts)
    each("prompt", None)
    for t in range(5):
        s.buf.decode_step(*s.inputs(10 + 2 * t))
    each("steps", None)
    keep = pick(KEEP)
    if alone:
        if keep[0]:
            s.commit(2, [4], [pick(PATH)[0][:keep[0]]])
    else:
        s.commit(2, [4] * len(s.which), pick(PATH), keep)
    each("drafts", None)
    for t in range(4):
        s.buf.decode_step(*s.inputs(30 + 2 * t))
    each("more steps", None)
    q, k, v = s.inputs(50)
    L = s.buf.kv.len + 1
    scores = torch.full((s.buf.U, L), float("nan"), device="cuda")
    if units and not alone:
        s.buf.decode_evict_units(pol, torch.full((s.buf.U,), budget, dtype=torch.int32, device="cuda"), budget, q, k, v,
                                 scores_out=scores)
    elif units:
        s.buf.decode_evict(pol, budget, q, k, v, scores_out=scores)
    else:
        s.buf.decode_step(q, k, v)
        s.buf.score_evict(pol, budget, scores_out=scores)
    each("evicted", scores)
    for t in range(4):
        s.buf.decode_step(*s.inputs(60 + 2 * t))
    each("steps on the rest", None)


def _compare(batch, look, hk, G, D, window, policy, units, budget, prompt=PROMPT):
    hidden, n_in, ln = policy
    params = _params(hidden, n_in, ln)
    pol, cap = make_policy(params, hidden, n_in, ln), max(prompt) + 30
    names = ["k", "v", "alpha", "num", "den", "vnorm"] + (["sigma"] if n_in == 5 else [])
    got, want = {}, {}
    s = Sequences(list(range(batch)), hk, G, D, window, True, n_in == 5, cap)

    def keep_batch(stage, scores):
        for b in look:
            got[stage, b] = s.state(b)
            if scores is not None:
                got["scores", b] = scores[b * hk:(b + 1) * hk].cpu().double().numpy()
    _run(s, prompt, budget, pol, units, keep_batch)
    for b in look:
        one = Sequences([b], hk, G, D, window, False, n_in == 5, cap)

        def keep_one(stage, scores):
            want[stage, b] = one.state(b) if one.buf.kv.len else []
            if scores is not None:
                want["scores", b] = scores.cpu().double().numpy()
        _run(one, prompt, budget, pol, units, keep_one)
        n = prompt[b % 5] + KEEP[b % 5] + 10
        for stage in ("prompt", "steps", "drafts", "more steps"):
            assert want[stage, b] or (stage == "prompt" and prompt[b % 5] == 0)
            _same(got[stage, b], want[stage, b], names, (b, stage))
        for h in range(hk):
            assert want["more steps", b][h]["pos"].tolist() == list(range(n - 1))
            mine, theirs = got["scores", b][h][:n], want["scores", b][h][:n]
            ok, worst = H.vec_ok(mine, theirs, tol=2 * H.FP_TOL)
            assert ok, (b, h, worst)
            keep = set(got["evicted", b][h]["pos"].astype(int))
            assert keep == set(osel.top_budget(mine, np.arange(n), budget).tolist()), (b, h)
            order = np.sort(theirs)[::-1]
            if n > budget and order[budget - 1] - order[budget] > 4 * H.FP_TOL * np.abs(theirs).max():
                assert keep == set(want["evicted", b][h]["pos"].astype(int)), (b, h)
        if all(np.array_equal(x["pos"], y["pos"]) for x, y in zip(got["evicted", b], want["evicted", b])):
            _same(got["steps on the rest", b], want["steps on the rest", b], names, (b, "steps on the rest"))


@pytest.mark.parametrize("policy", POLICIES)
@pytest.mark.parametrize("G,D,window", [(4, 128, 3), (2, 64, 6)])
def test_a_sequence_of_an_uneven_batch_is_as_alone(policy, G, D, window):
    # prompts of different lengths (one empty), accepted paths of different lengths between the steps of
    # the entropy window, an eviction: positions, features and scores do not depend on the neighbours
    _compare(5, range(5), 2, G, D, window, policy, False, 16)


@pytest.mark.parametrize("G,window", [(4, 3), (8, 5), (2, 4)])
def test_a_sequence_of_a_large_uneven_batch_is_as_alone(G, window):
    # enough units for the launch of a whole ragged step with per-unit budgets
    _compare(80, [0, 1, 2, 3, 4, 77, 79], 2, G, 128, window, POLICIES[0], True, 16)


def test_a_long_sequence_among_short_ones_is_as_alone():
    # units that fit on chip and the chunks of longer ones share a launch
    _compare(80, [0, 1, 2, 5], 2, 4, 128, 3, POLICIES[0], True, 16, [6000, 7, 0, 23, 31])


def test_the_window_of_an_uneven_batch_against_the_oracle():
    # one sequence of three, step by step in binary64: the terms of steps before and after a commit of
    # uneven paths leave the window as they came
    s = Sequences([0, 1, 2], 1, 4, 128, 3, True, False, 60)
    counts, keep, path = [21, 9, 14], [1, 3, 0], [[2, 3, 3], [0, 2, 3], [0, 1, 2]]
    b = 1
    s.commit(1, counts)
    rows = H.to_np(s.rows(1, b, 9)).astype(np.float64)[:, 0]
    st = ounit.new_student(rows[0], rows[1], np.arange(9), G=4, scale=128 ** -0.5, window=3)
    for t in range(9):
        if t == 4:
            s.commit(2, [4, 4, 4], path, keep)
            new = H.to_np(s.rows(2, b, 4)).astype(np.float64)[:, 0]
            for j in path[b][:keep[b]]:
                ounit._append(st, new[0, j], new[1, j])
                st.alpha, st.N, st.Z = (np.append(x, 0.0) for x in (st.alpha, st.N, st.Z))
                st.hist.append_rows(1)
        q, k, v = s.inputs(10 + 2 * t)
        s.buf.decode_step(q, k, v)
        ounit.decode_step(st, *(H.to_np(x[b]).astype(np.float64) for x in (q, k, v)))
        got = s.state(b)[0]
        Z, N = st.hist.sums()
        assert got["pos"].tolist() == st.pos.tolist(), t
        for name, ref in (("alpha", st.alpha), ("num", N), ("den", Z)):
            ok, worst = H.vec_ok(got[name], ref)
            assert ok, (t, name, worst)


def test_replays_of_an_uneven_commit_repeat_it():
    # the row of the table that a commit writes is not the one it reads
    s = Sequences([0, 1, 2], 2, 4, 128, 3, True, False, 60)
    s.commit(1, [20, 5, 11])
    n, nxt, at = s.buf.kv.len, s.buf.feat.next_pos, s.buf.feat.behind_row
    lens = s.buf.unit_len.clone()
    t = make_tokens([3, 3, 3])
    keep = torch.tensor([1, 3, 2], dtype=torch.int32, device="cuda")

    def step():
        s.buf.kv.len, s.buf.feat.next_pos = n, nxt
        s.buf.feat.behind_row, s.buf.feat.behind_at = at, nxt
        s.buf.unit_len.copy_(lens)
        s.buf.commit_rows(t, keep=keep)

    step()
    want = [x.clone() for x in (s.buf.pos, s.buf.behind, s.buf.unit_len)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        s.buf.pos.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        for u, (r, b) in enumerate(zip(lens.tolist(), [0, 0, 1, 1, 2, 2])):
            first = [20, 5, 11][b]
            assert s.buf.pos[u, r:r + [1, 3, 2][b]].tolist() == list(range(first, first + [1, 3, 2][b]))
        assert torch.equal(s.buf.behind, want[1]) and torch.equal(s.buf.unit_len, want[2])
        step()
