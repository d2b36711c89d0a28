"""Several tokens at once on the GPU against the binary64 oracle: norm and rotation of heads,
prompt and tree attention, commit of rows, and a run of them together.

Tolerances count roundings.  H = half a step of the output's type (finfo.eps / 2), F that of
float32.  Rotated heads: the store H |y|; in float32 the norm (at most D + 8 roundings of the sum
of squares, halved by the root, and the two products) and the rotation (two products and a sum, the
angle and its sine within 4 F) stay within (D / 2 + 16) F of the pair's magnitude.  Attention with
weights a_i: the store H |o|; every weight off by 2 E relative, E the error of its logit, which is
(D + 8) F scale sum |q_e k_e| at most, plus 8 F for the exponential, plus (keys) F for the sums:
(...) sum a_i |v_i|.  In bf16 also by its own rounding before it meets the values, by d_i <= H relative; the
sum that divides is that of the rounded weights, so to first order the output moves by
sum a_i d_i (v_i - o) <= H (sum a_i |v_i| + |o|)."""
import numpy as np
import pytest
import torch

from oracle import prompt as op
from oracle import select as osel
from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers, make_policy, make_rope, make_tokens

pytestmark = pytest.mark.gpu

F = torch.finfo(torch.float32).eps / 2
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def np64(t):
    return t.detach().double().cpu().numpy()


class Cache:
    """A cache with random rows everywhere, per-unit lengths if given, and its units' sequences."""

    def __init__(self, counts, rows, dtype="bf16", D=128, hk=2, G=4, layers=1, lens=None, spare=3, seed=0,
                 features=False, sigma=False, ragged=None):
        g = torch.Generator().manual_seed(seed)
        self.B, self.hk, self.G, self.D, self.layers, self.dtype = len(counts), hk, G, D, layers, dtype
        self.counts, self.td = counts, TYPES[dtype]
        U = self.B * layers * hk
        cap = rows + max(counts) + spare
        self.buf = DecodeBuffers(self.B, layers, hk * G, hk, D, cap, dtype, features=features, sigma=sigma,
                                 ragged=lens is not None if ragged is None else ragged)
        self.lens = list(lens) if lens is not None else [rows] * U
        self.buf.k.copy_(torch.randn((U, cap, D), generator=g).to(self.td))
        self.buf.v.copy_(torch.randn((U, cap, D), generator=g).to(self.td))
        self.buf.kv.len = rows
        if self.buf.unit_len is not None:
            self.buf.unit_len.copy_(torch.tensor(self.lens, dtype=torch.int32))
        self.tokens = make_tokens(counts)
        self.N = sum(counts)
        self.q = torch.randn((self.N, hk * G, D), generator=g).to(self.td).cuda()
        self.g = g

    def unit(self, b, layer, h):
        return (b * self.layers + layer) * self.hk + h

    def spans(self):
        at = 0
        for b, n in enumerate(self.counts):
            yield b, at, n
            at += n


def check_attention(c, out, layer, masks):
    """out against the oracle, every sequence and KV head; masks[b] (n, n)."""
    scale = 1 / np.sqrt(c.D)
    H = half_step(c.dtype)
    q, o = np64(c.q), np64(out)
    for b, at, n in c.spans():
        if n == 0:
            continue
        for h in range(c.hk):
            u = c.unit(b, layer, h)
            r = c.lens[u]
            K, V = np64(c.buf.k[u, :r + n]), np64(c.buf.v[u, :r + n])
            see = np.concatenate([np.ones((n, r), bool), masks[b]], 1)
            K, V = np.where(see.any(0)[:, None], K, 0), np.where(see.any(0)[:, None], V, 0)
            x = q[at:at + n, h * c.G:(h + 1) * c.G]
            s = np.where(see[:, None], scale * np.einsum("ngd,kd->ngk", x, K), -np.inf)
            mag = scale * np.einsum("ngd,kd->ngk", np.abs(x), np.abs(K)).max(-1, keepdims=True)
            e = np.exp(s - s.max(-1, keepdims=True))
            a = e / e.sum(-1, keepdims=True)
            ref = a @ V
            off = 2 * ((c.D + 8) * F * mag + 8 * F) + (r + n) * F + (H if c.dtype == "bf16" else 0)
            tol = (2 if c.dtype == "bf16" else 1) * H * np.abs(ref) + off * (a @ np.abs(V)) + 1e-30
            got = o[at:at + n, h * c.G:(h + 1) * c.G]
            bad = ~(np.abs(got - ref) <= tol)
            assert not bad.any(), (b, h, np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4], tol[bad][:4])
            for t in {0, n - 1}:                 # the vectorised reference is the oracle's loop
                one = op.attend_tokens(x[t:t + 1], K[see[t]], V[see[t]], int(see[t].sum()) - 1, np.ones((1, 1), bool),
                                       scale)
                assert np.allclose(one[0], ref[t], rtol=1e-10, atol=1e-10)


def close(got, want, keys, vmax, dtype):
    """The same sums cut and ordered otherwise.  Each side is off by the store's rounding H |o|, that of
    `keys` float32 terms, (keys + 8) F vmax, and in bf16 by the rounding of its weights before they meet
    the values: exp(s - m) is rounded against the maximum m of the keys met so far, which differs with
    the cut, so up to H (sum a_i |v_i| + |o|) <= 2 H vmax on either side."""
    got, want = np64(got), np64(want)
    H = half_step(dtype)
    off = (keys + 8) * F * vmax + (2 * H * vmax if dtype == "bf16" else 0)
    return np.all(np.abs(got - want) <= 2 * (H * np.abs(want) + off))


def random_tree(n, seed):
    g = np.random.default_rng(seed)
    return [int(g.integers(-1, i)) if i else -1 for i in range(n)]


def uneven(units, rows):
    return [max(0, rows - (5 * i) % 7 * (rows // 9)) for i in range(units)]


# ------------------------------------------------------------------------ norm and rotation

def rope_case(c, layer, rot, inter, norm, far, cache, gains=True, ragged_ld=True):
    hk, hq, D, N = c.hk, c.hk * c.G, c.D, c.N
    wide = (hq + 2 * hk) * D + (16 if ragged_ld else 0)
    qkv = torch.randn((N, wide), generator=c.g).to(c.td).cuda()
    q, k, v = qkv[:, :hq * D].unflatten(1, (hq, D)), qkv[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D)), \
        qkv[:, (hq + hk) * D:(hq + 2 * hk) * D].unflatten(1, (hk, D))
    pos = torch.randint(-5 if far else 0, far + 1, (N,), generator=c.g, dtype=torch.int32).cuda()
    f = torch.tensor([10000.0 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float32).cuda() if rot else None
    gq, gk = ((1 + 0.2 * torch.randn(D, generator=c.g)).cuda() for _ in range(2)) if gains else (None, None)
    rope = make_rope(f, inter, norm, 1e-5, gq, gk)
    k0, v0 = c.buf.k.clone(), c.buf.v.clone()
    qo, ko = c.buf.norm_rope(c.tokens, rope, q, k, v if cache else None, pos if rot else None, layer)
    torch.cuda.synchronize()
    ref = {}
    for name, x, gain, got in (("q", q, gq, qo), ("k", k, gk, ko)):
        fr = np64(f) if rot else None
        y = op.norm_rope(np64(x), pos.cpu().numpy(), fr, np64(gain) if gains else None, norm, float(np.float32(1e-5)),
                         inter)
        pre = op.norm_rope(np64(x), pos.cpu().numpy(), None, np64(gain) if gains else None, norm,
                           float(np.float32(1e-5)))
        mag = np.abs(pre)
        if rot:
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
            pair = np.hypot(pre[..., a], pre[..., b])
            mag[..., a] = mag[..., b] = pair
        ref[name] = (y, half_step(c.dtype) * np.abs(y) + (D / 2 + 16) * F * mag)
        if got is not None:
            assert np.all(np.abs(np64(got) - y) <= ref[name][1]), name
    if not cache:
        assert torch.equal(k0, c.buf.k) and torch.equal(v0, c.buf.v)
        return
    assert ko is None
    kc, vc = np64(c.buf.k), np64(c.buf.v)
    touched = np.zeros(kc.shape[:2], bool)
    for b, at, n in c.spans():
        for h in range(hk):
            u = c.unit(b, layer, h)
            r = c.lens[u]
            touched[u, r:r + n] = True
            y, tol = (z[at:at + n, h] for z in ref["k"])
            assert np.all(np.abs(kc[u, r:r + n] - y) <= tol)
            assert np.array_equal(vc[u, r:r + n], np64(v)[at:at + n, h])
    assert np.array_equal(kc[~touched], np64(k0)[~touched]) and np.array_equal(vc[~touched], np64(v0)[~touched])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rot,inter,norm,far", [(-1, False, True, 5000), (-1, True, True, 1 << 20), (-2, False, False, 90),
                                                (16, True, False, 300), (16, False, True, 2**31 - 2), (0, False, True, 0),
                                                (48, False, True, 700)])
def test_norm_rope(dtype, D, rot, inter, norm, far):
    rot = {-1: D, -2: D // 2}.get(rot, rot)
    for counts, hk, G, layers, lens in (([1], 1, 1, 1, None), ([5, 0, 3], 2, 4, 2, 11), ([2, 2], 3, 8, 1, None)):
        lens = uneven(len(counts) * layers * hk, 11) if lens else None
        print(f"norm_rope {dtype} D={D} rot={rot} inter={inter} counts={counts}", flush=True)
        for cache in (False, True):
            c = Cache(counts, 11, dtype, D, hk, G, layers, lens, seed=rot + D)
            rope_case(c, layers - 1, rot, inter, norm, far, cache, gains=inter or far > 90)


@pytest.mark.parametrize("counts,dtype,D,hk,G", [([8001, 0, 8195, 300], "bf16", 64, 1, 2),
                                                 ([1700, 1306], "f32", 128, 8, 4)])
def test_norm_rope_of_many_tokens(counts, dtype, D, hk, G):
    # over the size from which a workgroup takes several tokens
    c = Cache(counts, 0, dtype, D, hk, G, seed=5, lens=[0] * (len(counts) * hk))
    rope_case(c, 0, D, False, True, 9000, True)
    rope_case(c, 0, D // 2, True, True, 9000, False)


def test_norm_rope_in_place_and_single_heads():
    c = Cache([3], 4, "f32", 64, 1, 1, seed=3)
    x = torch.randn((3, 1, 64), generator=c.g).cuda()
    f = torch.rand(32, generator=c.g).cuda()
    pos = torch.tensor([0, 7, 3], dtype=torch.int32, device="cuda")
    rope = make_rope(f, norm=True)
    want, _ = c.buf.norm_rope(c.tokens, rope, x, x.clone(), None, pos)
    y, z = x.clone(), x.clone()
    c.buf.norm_rope(c.tokens, rope, y, z, None, pos, q_out=y, k_out=z)
    assert torch.equal(y, want) and torch.equal(z, want)


def test_zero_rows_and_infinite_elements():
    c = Cache([4], 2, "bf16", 128, 1, 1, seed=4)
    x = torch.randn((4, 1, 128), generator=c.g).to(torch.bfloat16).cuda()
    x[1] = 0
    x[2, 0, 5] = float("inf")
    x[3, 0, 5] = float("nan")
    rope = make_rope(torch.rand(64, generator=c.g).cuda(), norm=True)
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    y, _ = c.buf.norm_rope(c.tokens, rope, x, x.clone(), None, pos)
    assert torch.isfinite(y[:2]).all() and (y[1] == 0).all()
    assert torch.isnan(y[2, 0, 5]) and torch.isnan(y[3]).all()


# ------------------------------------------------------------------------ prompt attention

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,hk,G", [(128, 2, 4), (64, 1, 8), (128, 3, 1), (64, 2, 2)])
@pytest.mark.parametrize("counts,rows,lens", [
    ([1], 0, False), ([1, 1], 700, False), ([33, 0, 1, 130], 0, False), ([5, 2], 2100, True), ([257], 63, False),
    ([64, 31, 128], 129, True)])
def test_prompt_attention(dtype, D, hk, G, counts, rows, lens):
    print(f"prompt {dtype} D={D} hk={hk} G={G} counts={counts} rows={rows}", flush=True)
    layers = 2 if lens else 1
    c = Cache(counts, rows, dtype, D, hk, G, layers,
              uneven(len(counts) * layers * hk, rows) if lens else None, seed=rows + D)
    out = c.buf.prompt_attention(c.tokens, c.q, layers - 1)
    check_attention(c, out, layers - 1, [op.causal_mask(n) for n in counts])


# Calls with enough workgroups for the tiles of 128 rows and of 64 (bf16, up to 64 rows of a
# sequence and KV head), whole and in parts of the key range, as prompts and as trees.
MANY = [([130, 0, 97, 40] * 3 + [33], 70, 8, 4, False), ([16, 3, 1, 9] * 5, 290, 8, 4, True),
        ([300, 17], 900, 8, 8, False), ([60] * 9, 0, 8, 1, False)]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("counts,rows,hk,G,lens", MANY)
def test_many_rows(dtype, D, tree, counts, rows, hk, G, lens):
    if tree and max(counts) > 256:
        counts = [256, 17]
    print(f"many rows {dtype} D={D} tree={tree} counts={counts[:4]}", flush=True)
    c = Cache(counts, rows, dtype, D, hk, G, 1, uneven(len(counts) * hk, rows) if lens else None, seed=rows + D)
    if tree:
        parents = [random_tree(n, 5 * b + n) for b, n in enumerate(counts)]
        flat = torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda")
        check_attention(c, c.buf.tree_attention(c.tokens, flat, c.q), 0, [op.tree_mask(p) for p in parents])
    else:
        check_attention(c, c.buf.prompt_attention(c.tokens, c.q), 0, [op.causal_mask(n) for n in counts])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("counts,rows,hk,G,lens", MANY)
def test_many_rows_do_not_depend_on_unseen_values(dtype, D, counts, rows, hk, G, lens):
    c = Cache(counts, rows, dtype, D, hk, G, 1, uneven(len(counts) * hk, rows) if lens else None, seed=rows + D)
    want = c.buf.prompt_attention(c.tokens, c.q)
    at = [(b, t0, n // 2) for b, t0, n in c.spans() if n > 1]
    for b, t0, r in at:
        for h in range(hk):
            u = c.unit(b, 0, h)
            c.buf.v[u, c.lens[u] + r:] = float("inf") if h % 2 else float("nan")
            c.buf.k[u, c.lens[u] + r:] = float("nan") if h % 2 else -float("inf")
    got = c.buf.prompt_attention(c.tokens, c.q)
    for b, t0, r in at:
        assert close(got[t0:t0 + r], want[t0:t0 + r], rows + max(counts), 6, dtype), b
        assert not torch.isfinite(got[t0 + r].float()).any()


def test_a_query_that_is_not_a_number_stays_alone():
    for dtype in ("bf16", "f32"):
        c = Cache([50], 100, dtype, 128, 2, 4, seed=14)
        want = c.buf.prompt_attention(c.tokens, c.q)
        c.q[7, 3, 5] = float("nan")
        c.q[9, 6] = float("inf")
        got = c.buf.prompt_attention(c.tokens, c.q)
        assert torch.isnan(got[7, 3]).all() and torch.isnan(got[9, 6]).all()
        got[7, 3], got[9, 6] = want[7, 3], want[9, 6]
        assert close(got, want, 150, 6, dtype)


def test_a_scale_of_its_own():
    c = Cache([21], 60, "bf16", 64, 2, 2, seed=15)
    base = c.buf.prompt_attention(c.tokens, c.q)
    c.buf.dims.scale = 0.25
    got = c.buf.prompt_attention(c.tokens, c.q)
    c.q = (c.q.float() * 2).to(c.td)                # 0.25 = 2 / sqrt(64): powers of two, exact
    c.buf.dims.scale = 0.0
    assert torch.equal(got, c.buf.prompt_attention(c.tokens, c.q)) and not torch.equal(got, base)


def test_a_cache_past_the_memory_side_cache():
    # over 256 MB of rows that are read once: other loads
    c = Cache([5], 70000, "bf16", 128, 8, 4, seed=16)
    check_attention(c, c.buf.prompt_attention(c.tokens, c.q), 0, [op.causal_mask(5)])
    c = Cache([16], 70000, "f32", 64, 8, 4, seed=17)
    p = random_tree(16, 3)
    check_attention(c, c.buf.tree_attention(c.tokens, torch.tensor(p, dtype=torch.int32, device="cuda"), c.q), 0,
                    [op.tree_mask(p)])


def test_prompt_attention_does_not_depend_on_unseen_rows():
    # value and key rows that a token does not see: infinite, NaN and the largest numbers
    for dtype in ("bf16", "f32"):
        c = Cache([40], 70, dtype, 128, 1, 4, seed=8, spare=200)
        want = c.buf.prompt_attention(c.tokens, c.q)
        r = 70 + 17
        for x, y in ((float("nan"), float("inf")), (float("inf"), float("nan")), (3e38, -float("inf"))):
            c.buf.k[:, r:] = x
            c.buf.v[:, r:] = y
            got = c.buf.prompt_attention(c.tokens, c.q)
            assert close(got[:17], want[:17], 110, 6, dtype), (dtype, x)
            assert not torch.isfinite(got[17:].float()).any()
        # what is seen is as the formula has it
        c.buf.k[:, r:], c.buf.v[:, r:] = 0, 1
        c.buf.v[:, r + 3, 5] = float("inf")
        got = c.buf.prompt_attention(c.tokens, c.q).float()
        assert torch.isinf(got[20:, :, 5]).all() and torch.isfinite(got[:20]).all()
        got[20:, :, 5] = 0
        assert torch.isfinite(got).all()


def test_rows_behind_the_tokens_and_other_outputs_are_left():
    c = Cache([3, 1, 2], 300, "bf16", 128, 2, 4, seed=9, spare=60, lens=uneven(6, 300))
    k0, v0 = c.buf.k.clone(), c.buf.v.clone()
    out = torch.full((c.N + 2, c.hk * c.G, c.D), 7.0, dtype=c.td, device="cuda")
    c.buf.prompt_attention(c.tokens, c.q, out=out[1:-1])
    c.buf.tree_attention(c.tokens, torch.full((c.N,), -1, dtype=torch.int32, device="cuda"), c.q, out=out[1:-1])
    assert (out[0] == 7).all() and (out[-1] == 7).all()
    assert torch.equal(k0, c.buf.k) and torch.equal(v0, c.buf.v)


def test_extreme_logits():
    # one key far above the others: all weight on it; then all keys equal
    for dtype in ("bf16", "f32"):
        c = Cache([40], 1000, dtype, 64, 1, 2, seed=10)
        c.q.fill_(8.0)
        c.buf.k.zero_()
        c.buf.k[0, 500] = 100.0
        out = c.buf.prompt_attention(c.tokens, c.q).float()
        # out = fl(fl(p v) fl(1 / p)) for the one weight p that is left: three roundings, and in
        # bf16 the store then finds v again
        v = np64(c.buf.v[0, 500])
        assert np.all(np.abs(np64(out) - v) <= (0 if dtype == "bf16" else 3.01 * F) * np.abs(v))
        c.buf.k.fill_(-1000.0)
        check_attention(c, c.buf.prompt_attention(c.tokens, c.q), 0, [op.causal_mask(40)])


def test_offsets_past_32_bits():
    # the last unit's rows start 4 GiB and more behind the buffers' start
    cap, D = (1 << 21) + 40, 128
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB")
    c = Cache([3], 30, "bf16", D, 1, 4, seed=11)
    big = DecodeBuffers(1, 9, 4, 1, D, cap, features=False)
    big.kv.len = cap - 3
    u = 8
    assert u * cap * D * 2 > 1 << 32
    c.q.abs_()
    big.k[u], big.v[u] = -1000.0, 7.0          # far below the last rows' logits: no weight at all
    big.k[u, cap - 33:] = c.buf.k[0, :33]
    big.v[u, cap - 33:] = c.buf.v[0, :33]
    rope, pos = make_rope(torch.rand(64, generator=c.g).cuda()), torch.arange(3, dtype=torch.int32, device="cuda")
    kk, vv = (torch.randn((3, 1, D), generator=c.g).to(torch.bfloat16).cuda() for _ in range(2))
    for b in (big, c.buf):
        b.norm_rope(c.tokens, rope, c.q, kk, vv, pos, layer=8 if b is big else 0)
    assert torch.equal(big.k[u, cap - 3:], c.buf.k[0, 30:33]) and torch.equal(big.v[u, cap - 3:], c.buf.v[0, 30:33])
    assert close(big.prompt_attention(c.tokens, c.q, 8), c.buf.prompt_attention(c.tokens, c.q), 33, 6, "bf16")
    chain = torch.arange(-1, 2, dtype=torch.int32, device="cuda")
    assert close(big.tree_attention(c.tokens, chain, c.q, 8), c.buf.prompt_attention(c.tokens, c.q), 33, 6, "bf16")
    path = torch.tensor([[1, 2]], dtype=torch.int32, device="cuda")
    want = big.k[u, cap - 2:].clone()
    big.commit_rows(c.tokens, path)
    assert torch.equal(big.k[u, cap - 3:cap - 1], want) and big.kv.len == cap - 1


# ------------------------------------------------------------------------ tree attention

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,hk,G", [(128, 2, 4), (64, 1, 8), (64, 3, 1)])
@pytest.mark.parametrize("counts,rows,lens", [
    ([1], 0, False), ([7], 33, False), ([13], 4097, False), ([8, 0, 33, 1], 300, True), ([256, 65], 70, False),
    ([64], 0, False), ([32, 31], 1500, True)])
def test_tree_attention(dtype, D, hk, G, counts, rows, lens):
    print(f"tree {dtype} D={D} hk={hk} G={G} counts={counts} rows={rows}", flush=True)
    c = Cache(counts, rows, dtype, D, hk, G, 1, uneven(len(counts) * hk, rows) if lens else None, seed=rows + D + 1)
    parents = [random_tree(n, 17 * b + n) for b, n in enumerate(counts)]
    flat = torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda")
    out = c.buf.tree_attention(c.tokens, flat, c.q)
    check_attention(c, out, 0, [op.tree_mask(p) for p in parents])


def test_a_chain_of_drafts_is_the_prompt():
    for n, rows in ((256, 0), (31, 40), (5, 900)):
        c = Cache([n], rows, "bf16", 128, 2, 4, seed=n)
        chain = torch.arange(-1, n - 1, dtype=torch.int32, device="cuda")
        assert torch.equal(c.buf.tree_attention(c.tokens, chain, c.q), c.buf.prompt_attention(c.tokens, c.q))


def test_parents_that_are_no_earlier_node_count_as_none():
    c = Cache([6], 50, "bf16", 128, 1, 4, seed=12)
    odd = torch.tensor([0, 5, 1, 2**31 - 1, -2**31, 4], dtype=torch.int32, device="cuda")
    out = c.buf.tree_attention(c.tokens, odd, c.q)
    check_attention(c, out, 0, [op.tree_mask([-1, -1, 1, -1, -1, 4])])


def test_tree_attention_does_not_depend_on_other_branches():
    c = Cache([9], 20, "bf16", 64, 1, 2, seed=13)
    parent = [-1, 0, 0, 1, 2, 3, 4, 5, 6]            # 0-1-3-5-7 and 0-2-4-6-8
    p = torch.tensor(parent, dtype=torch.int32, device="cuda")
    want = c.buf.tree_attention(c.tokens, p, c.q)
    c.buf.k[0, 22], c.buf.v[0, 22] = float("nan"), float("inf")           # node 2
    got = c.buf.tree_attention(c.tokens, p, c.q)
    sees = op.tree_mask(parent)[:, 2]
    for i in range(9):
        assert close(got[i], want[i], 29, 6, "bf16") if not sees[i] else not torch.isfinite(got[i].float()).any()


# ------------------------------------------------------------------------ commit

@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("with_path,with_keep", [(False, False), (True, False), (True, True), (False, True)])
def test_commit_rows(dtype, D, with_path, with_keep):
    counts, rows, layers, hk = [70, 3, 0, 41], 30, 2, 2
    U = 4 * layers * hk
    c = Cache(counts, rows, dtype, D, hk, 2, layers, uneven(U, rows), seed=D, features=True, sigma=True)
    buf = c.buf
    for x in (buf.alpha, buf.num, buf.den, buf.vnorm, buf.sigma):
        x.copy_(torch.rand(x.shape, generator=c.g, dtype=x.dtype))
    buf.feat.next_pos = 500
    g = np.random.default_rng(D)
    width = 37 if with_path else 70
    path = np.sort(g.choice(70, (4, width)), 1) if with_path else None
    if with_path:
        path[0] = np.arange(width) + 33                  # every row moves into one that another pass has read
        path[3, :5] = [-7, 40, 0, 2**31 - 1, -2**31]     # clamped
    keep = [50, 9, 4, -3] if with_keep else None
    before = {n: np64(x) for n, x in (("k", buf.k), ("v", buf.v), ("alpha", buf.alpha), ("num", buf.num),
                                      ("den", buf.den), ("pos", buf.pos), ("vnorm", buf.vnorm), ("sigma", buf.sigma))}
    dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    buf.commit_rows(c.tokens, dev(path), dev(keep))
    torch.cuda.synchronize()
    assert buf.kv.len == rows + width and buf.feat.next_pos == 500 + width
    want = {n: x.copy() for n, x in before.items()}
    lens = []
    for u in range(U):
        b, r = u // (layers * hk), c.lens[u]
        src = op.kept_rows(counts[b], None if path is None else path[b], None if keep is None else keep[b], width)
        for j, t in enumerate(src):
            want["k"][u, r + j], want["v"][u, r + j] = before["k"][u, r + t], before["v"][u, r + t]
            for n in ("alpha", "num", "den", "sigma"):
                want[n][u, r + j] = 0
            want["pos"][u, r + j] = 500 + j
            want["vnorm"][u, r + j] = np.linalg.norm(before["v"][u, r + t])
        lens.append(r + len(src))
    assert buf.unit_len.tolist() == lens
    for n, x in want.items():
        got = np64(getattr(buf, n))
        if n == "vnorm":                                  # D + 2 roundings in float32, halved by the root
            assert np.all(np.abs(got - x) <= (D / 2 + 3) * F * np.abs(x))
        else:
            assert np.array_equal(got, x), n


def test_commit_on_a_uniform_cache_without_features():
    c = Cache([4, 4], 10, "bf16", 128, 1, 4, seed=20)
    k0 = c.buf.k.clone()
    c.buf.commit_rows(c.tokens, torch.tensor([[0, 2], [1, 3]], dtype=torch.int32, device="cuda"))
    assert c.buf.kv.len == 12
    k0[0, 11], k0[1, 10], k0[1, 11] = c.buf.k[0, 11], k0[1, 11].clone(), k0[1, 13].clone()
    assert torch.equal(k0, c.buf.k) and torch.equal(c.buf.k[0, 11], c.buf.k[0, 12])


def test_commit_as_feat_init():
    # a committed prompt leaves the state that dc_feat_init gives the same cache
    c = Cache([90], 0, "bf16", 128, 2, 4, seed=21, features=True, sigma=True)
    for x in (c.buf.alpha, c.buf.num, c.buf.den, c.buf.vnorm, c.buf.sigma):
        x.fill_(3)
    c.buf.commit_rows(c.tokens)
    got = [x[:, :90].clone() for x in (c.buf.alpha, c.buf.num, c.buf.den, c.buf.pos, c.buf.vnorm, c.buf.sigma)]
    nxt = c.buf.feat.next_pos
    c.buf.feat_init(90)
    for a, b in zip(got, (c.buf.alpha, c.buf.num, c.buf.den, c.buf.pos, c.buf.vnorm, c.buf.sigma)):
        assert torch.equal(a, b[:, :90])
    assert nxt == c.buf.feat.next_pos == 90


# ------------------------------------------------------------------------ together

def _projections(n, hq, hk, D, g):
    x = torch.randn((n, (hq + 2 * hk) * D), generator=g).to(torch.bfloat16).cuda()
    return [y.unflatten(1, (-1, D)) for y in x.split([hq * D, hk * D, hk * D], 1)]


def test_prompt_in_parts_drafts_and_evicting_steps():
    """Two packed prompts go in as a whole and in two parts; drafts follow, a path is accepted, then
    decode steps evict: at every point the cache holds the rows that one token at a time would have
    put there, and the attention is the oracle's over them."""
    g = torch.Generator().manual_seed(30)
    hk, G, D, layers = 2, 4, 128, 2
    hq, counts = hk * G, [150, 150]
    rope = make_rope(torch.tensor([1e4 ** (-i / 64) for i in range(64)], dtype=torch.float32, device="cuda"), norm=True,
                     q_gain=torch.ones(D, device="cuda"), k_gain=torch.ones(D, device="cuda"))

    def new():
        return DecodeBuffers(2, layers, hq, hk, D, 200, features=True)

    whole, parts = new(), new()
    first, rest = [60, 60], [90, 90]
    for layer in range(layers):
        q, k, v = _projections(300, hq, hk, D, g)
        pos = torch.arange(150, dtype=torch.int32, device="cuda").repeat(2)
        out = whole.prefill(make_tokens(counts), rope, q, k, v, pos, layer)
        pick = lambda lo, hi: torch.cat([torch.arange(lo, hi), torch.arange(150 + lo, 150 + hi)]).cuda()  # noqa: E731
        got = torch.empty_like(out)
        for lo, hi, n in ((0, 60, first), (60, 150, rest)):
            parts.kv.len = lo                           # one layer at a time: the length is the caller's
            i = pick(lo, hi)
            got[i] = parts.prefill(make_tokens(n), rope, q[i], k[i], v[i], pos[i], layer)
        # the same keys in another order of tiles: two roundings of the output and of the weights apart
        assert torch.allclose(out.float(), got.float(), rtol=4 * half_step("bf16"), atol=2e-2)
    parts.kv.len = 0
    parts.commit_rows(make_tokens(first))
    parts.commit_rows(make_tokens(rest))
    whole.commit_rows(make_tokens(counts))
    assert torch.equal(whole.k, parts.k) and torch.equal(whole.v, parts.v) and whole.kv.len == parts.kv.len == 150
    assert torch.equal(whole.pos, parts.pos) and torch.equal(whole.vnorm, parts.vnorm)

    # drafts: nodes 0, 1, 3 of each tree are accepted
    parent = [-1, 0, 0, 1, 2]
    flat = torch.tensor(parent * 2, dtype=torch.int32, device="cuda")
    depth = torch.tensor([150, 151, 151, 152, 152] * 2, dtype=torch.int32, device="cuda")
    t = make_tokens([5, 5])
    drafted = []
    for layer in range(layers):
        q, k, v = _projections(10, hq, hk, D, g)
        rq, rk = whole.norm_rope(t, rope, q, k, None, depth)
        out = whole.draft(t, flat, rope, q, k, v, depth, layer)
        drafted.append((rq, rk, v, out))
    path = torch.tensor([[0, 1, 3]] * 2, dtype=torch.int32, device="cuda")
    whole.commit_rows(t, path)
    # one token at a time on the other cache
    for step, node in enumerate((0, 1, 3)):
        qs, ks, vs = (torch.stack([torch.stack([d[x][b * 5 + node] for d in drafted]) for b in range(2)])
                      for x in range(3))
        o = parts.decode_step(qs.contiguous(), ks.contiguous(), vs.contiguous())
        for layer in range(layers):
            for b in range(2):
                assert torch.allclose(o[b, layer].float(), drafted[layer][3][b * 5 + node].float(),
                                      rtol=4 * half_step("bf16"), atol=2e-2)
    assert whole.kv.len == parts.kv.len == 153 and whole.feat.next_pos == parts.feat.next_pos
    assert torch.equal(whole.k[:, :153], parts.k[:, :153]) and torch.equal(whole.v[:, :153], parts.v[:, :153])
    assert torch.equal(whole.pos[:, :153], parts.pos[:, :153])
    assert torch.allclose(whole.vnorm[:, :153], parts.vnorm[:, :153], rtol=1e-5)

    # the cache then serves evicting steps
    params = (0.1 * torch.randn(4 * 32 + 32 + 32 + 1, generator=g)).cuda()
    U = 2 * layers * hk
    q = torch.randn((U, G, D), generator=g).to(torch.bfloat16).cuda()
    kn, vn = (torch.randn((U, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    scores = torch.empty((U, 154), device="cuda")
    whole.decode_evict(make_policy(params, (32,)), 64, q, kn, vn, scores_out=scores)
    assert whole.kv.len == 64
    for u in range(U):
        keep = osel.top_budget(scores[u].double().cpu().numpy(), np.arange(154), 64)
        assert set(whole.pos[u, :64].tolist()) == set(int(x) for x in keep)


def test_ragged_prompts_then_drafts_with_device_counts():
    g = torch.Generator().manual_seed(31)
    hk, G, D = 2, 4, 64
    hq, counts = hk * G, [40, 7, 33]
    buf = DecodeBuffers(3, 1, hq, hk, D, 128, features=True, ragged=True)
    rope = make_rope(torch.rand(32, generator=g).cuda())
    t = make_tokens(counts)
    q, k, v = _projections(80, hq, hk, D, g)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in counts]).cuda()
    buf.prefill(t, rope, q, k, v, pos)
    buf.commit_rows(t)
    lens = [n for n in counts for _ in range(hk)]
    assert buf.unit_len.tolist() == lens and buf.kv.len == 40
    t = make_tokens([4, 4, 4])
    q, k, v = _projections(12, hq, hk, D, g)
    pos = torch.tensor([n + d for n in counts for d in (0, 1, 1, 2)], dtype=torch.int32, device="cuda")
    parent = [-1, 0, 0, 2]
    rq, _ = buf.norm_rope(t, rope, q, k, None, pos)
    out = buf.draft(t, torch.tensor(parent * 3, dtype=torch.int32, device="cuda"), rope, q, k, v, pos)

    class C:
        pass
    c = C()
    c.D, c.G, c.hk, c.dtype, c.q, c.lens, c.counts, c.buf, c.layers = D, G, hk, "bf16", rq, lens, [4] * 3, buf, 1
    c.spans, c.unit = lambda: Cache.spans(c), lambda b, layer, h: Cache.unit(c, b, layer, h)
    check_attention(c, out, 0, [op.tree_mask(parent)] * 3)
    keep = torch.tensor([3, 0, 1], dtype=torch.int32, device="cuda")
    buf.commit_rows(t, torch.tensor([[0, 2, 3]] * 3, dtype=torch.int32, device="cuda"), keep)
    assert buf.unit_len.tolist() == [43, 43, 7, 7, 34, 34] and buf.kv.len == 43
    # and a decode step over the ragged cache
    o = buf.decode_step(torch.randn((6, G, D), generator=g).to(torch.bfloat16).cuda(),
                        *(torch.randn((6, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2)))
    assert torch.isfinite(o.float()).all() and buf.unit_len.tolist() == [44, 44, 8, 8, 35, 35]


def test_replayed_graph_and_other_streams_give_the_same_bits():
    g = torch.Generator().manual_seed(32)
    hk, G, D = 1, 4, 128
    buf = DecodeBuffers(1, 1, hk * G, hk, D, 3200, features=True, ragged=True)
    buf.k.copy_(torch.randn(buf.k.shape, generator=g).to(torch.bfloat16))
    buf.v.copy_(torch.randn(buf.v.shape, generator=g).to(torch.bfloat16))
    t = make_tokens([6])
    rope = make_rope(torch.rand(64, generator=g).cuda(), norm=True)
    q, k, v = (x.contiguous() for x in _projections(6, hk * G, hk, D, g))
    pos = torch.arange(3000, 3006, dtype=torch.int32, device="cuda")
    parent = torch.tensor([-1, 0, 0, 1, 3, 2], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 2, 5]], dtype=torch.int32, device="cuda")
    keep = torch.tensor([2], dtype=torch.int32, device="cuda")

    def step(out):
        buf.kv.len, buf.feat.next_pos = 3000, 3000
        buf.unit_len.fill_(2990)
        buf.draft(t, parent, rope, q, k, v, pos, out=out)
        buf.commit_rows(t, path, keep)

    want = torch.empty_like(q)
    step(want)
    torch.cuda.synchronize()
    kw, lw = buf.k.clone(), buf.unit_len.clone()
    side = torch.cuda.Stream()
    got = torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(got)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(buf.k, kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    for i in range(4):
        got.zero_()
        buf.unit_len.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(buf.k, kw) and torch.equal(buf.unit_len, lw), i
        step(torch.empty_like(want))                    # eager work between the replays


def test_offsets_that_are_no_partition_are_clamped():
    # counts over max_tokens, descending and negative offsets: nothing outside the arrays is touched
    c = Cache([4, 4, 4], 20, "bf16", 128, 1, 4, seed=40, lens=[20, 20, 20])
    t = make_tokens([4, 3, 4])
    t.tokens = 12
    for cu in ([0, 12, 3, 99], [-5, 2, 1, 12], [2**31 - 1, -2**31, 7, 8]):
        t.cu_tensor.copy_(torch.tensor(cu, dtype=torch.int32))
        out = torch.full((14, 4, 128), 5.0, dtype=c.td, device="cuda")
        q = torch.randn((12, 6 * 128), generator=c.g).to(c.td).cuda()
        a, b, d = (x.unflatten(1, (-1, 128)) for x in q.split([512, 128, 128], 1))
        c.buf.norm_rope(t, make_rope(), a, b, d)
        c.buf.prompt_attention(t, c.q, out=out[1:13])
        torch.cuda.synchronize()
        assert (out[0] == 5).all() and (out[13] == 5).all()


def test_wrappers_refuse():
    c = Cache([4, 4], 10, "bf16", 128, 1, 4, seed=41)
    buf, t = c.buf, c.tokens
    k = torch.zeros((8, 1, 128), dtype=c.td, device="cuda")
    p = torch.zeros(8, dtype=torch.int32, device="cuda")
    for bad in (c.q.float(), c.q[:7], c.q.transpose(1, 2), c.q.cpu(), c.q[:, :2]):
        with pytest.raises(ValueError):
            buf.norm_rope(t, make_rope(), bad, k)
        with pytest.raises(ValueError):
            buf.prompt_attention(t, bad)
        with pytest.raises(ValueError):
            buf.tree_attention(t, p, bad)
    with pytest.raises(ValueError):
        buf.tree_attention(t, p.long(), c.q)
    with pytest.raises(ValueError):
        buf.norm_rope(make_tokens([4]), make_rope(), c.q, k)
    with pytest.raises(ValueError):
        buf.commit_rows(t, torch.zeros((2, 2), device="cuda"))
    with pytest.raises(ValueError):
        make_rope(torch.zeros(64, dtype=torch.float64, device="cuda"))
    with pytest.raises(B.DCError):
        buf.commit_rows(t, keep=torch.ones(2, dtype=torch.int32, device="cuda"))   # a uniform cache
    with pytest.raises(B.DCError):
        buf.prompt_attention(t, c.q, layer=1)
    buf.kv.len = buf.cap - 3
    with pytest.raises(B.DCError):
        buf.prompt_attention(t, c.q)
