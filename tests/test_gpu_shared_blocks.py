"""Rows that sequences share and blocks of rows on the GPU against the binary64 oracle: shared attention, bounds,
choice of blocks, attention over chosen blocks, and a run of them together.

Bounds and choices are equal: a bound is one of the inputs, and scores are binary64 sums whose rounding,
2^-53 of the terms' magnitude for each of a few hundred, is far below the distance of two random scores; equal blocks
have equal scores on both sides.  Attention outputs stay within H |o| for the store and, with weights a_i,
E sum a_i |v_i| for the rest.  H is half a step of the output's type (finfo.eps / 2), F that of float32,
E = 2 ((D + 8) F scale sum |q_e k_e| + 8 F) + keys F, twice the relative error of a weight whose logit is off by its D
products and sums, the exponential, and the sums over the keys; in bf16 each weight is also rounded by d_i <= H
before it meets the values, and the sum that divides is that of the rounded ones: H (sum a_i |v_i| + |o|) more.
Joining the parts of the key range adds to the sums' roundings as keys do."""
import numpy as np
import pytest
import torch

from oracle import blocks as ob
from oracle import prompt as op
from paper_2608_08878_amd import binding as B
from paper_2608_08878_amd.buffers import DecodeBuffers, make_rope, make_shared, make_tokens

pytestmark = pytest.mark.gpu

F = torch.finfo(torch.float32).eps / 2
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(TYPES[dtype]).eps / 2


def np64(t):
    return t.detach().double().cpu().numpy()


def cache(batch, rows, lens, dtype="bf16", D=128, hk=2, G=4, layers=1, g=None, spare=3, ragged=True, magnitude=1.0):
    """A cache with random rows in every slot; lens per unit (None: rows each)."""
    U, cap = batch * layers * hk, rows + spare
    buf = DecodeBuffers(batch, layers, hk * G, hk, D, cap, dtype, features=False, ragged=ragged)
    buf.k.copy_(torch.randn((U, cap, D), generator=g).to(TYPES[dtype]))
    buf.v.copy_((magnitude * torch.randn((U, cap, D), generator=g)).to(TYPES[dtype]))
    buf.kv.len = rows
    if ragged:
        buf.unit_len.copy_(torch.tensor(lens if lens is not None else [rows] * U, dtype=torch.int32))
    return buf


def spans(counts):
    at = 0
    for b, n in enumerate(counts):
        yield b, at, n
        at += n


def attention_off(got, q, K, V, see, dtype):
    """Where got (n, G, d) is further from the oracle than the tolerance; K, V (keys, d), see (n, keys)."""
    D, H = K.shape[1], half_step(dtype)
    scale = 1 / np.sqrt(D)
    any_sees = see.any(0)[:, None]
    K, V = np.where(any_sees, K, 0), np.where(any_sees, V, 0)
    s = np.where(see[:, None], scale * np.einsum("ngd,kd->ngk", q, K), -np.inf)
    mag = scale * np.einsum("ngd,kd->ngk", np.abs(q), np.abs(K)).max(-1, keepdims=True)
    e = np.exp(s - s.max(-1, keepdims=True))
    a = e / e.sum(-1, keepdims=True)
    ref = a @ V
    off = 2 * ((D + 8) * F * mag + 8 * F) + see.shape[1] * F + (H if dtype == "bf16" else 0)
    tol = (2 if dtype == "bf16" else 1) * H * np.abs(ref) + off * (a @ np.abs(V)) + 1e-30
    one = op.attend_tokens(q[:1], K[see[0]], V[see[0]], int(see[0].sum()) - 1, np.ones((1, 1), bool), scale)
    assert np.allclose(one[0], ref[0], rtol=1e-10, atol=1e-10)      # the vectorised reference is the oracle's loop
    bad = ~(np.abs(got - ref) <= tol)
    return [(tuple(i), got[tuple(i)], ref[tuple(i)], tol[tuple(i)]) for i in np.argwhere(bad)[:4]]


def mask_of(parent, at, n):
    return op.causal_mask(n) if parent is None else op.tree_mask(parent[at:at + n])


def check_shared(out, buf, pre, counts, members, lens, plens, q, dtype, parent=None, layer=0):
    d = buf.dims
    hk, G, L = d.n_kv_heads, buf.G, d.n_layers
    first = np.concatenate([[0], np.cumsum(members)])
    o, x = np64(out), np64(q)
    for b, at, n in spans(counts):
        p = int(np.searchsorted(first, b, side="right")) - 1
        for h in range(hk if n else 0):
            u, r = (b * L + layer) * hk + h, lens[(b * L + layer) * hk + h]
            K, V = np64(buf.k[u, :r + n]), np64(buf.v[u, :r + n])
            before = r
            if p < len(members):
                pu = (p * L + layer) * hk + h
                K = np.concatenate([np64(pre.k[pu, :plens[pu]]), K])
                V = np.concatenate([np64(pre.v[pu, :plens[pu]]), V])
                before += plens[pu]
            see = np.concatenate([np.ones((n, before), bool), mask_of(parent, at, n)], 1)
            bad = attention_off(o[at:at + n, h * G:(h + 1) * G], x[at:at + n, h * G:(h + 1) * G], K, V, see, dtype)
            assert not bad, (b, h, bad)


def shared_case(counts, members, plen, rows, dtype="bf16", D=128, hk=2, G=4, layers=1, uneven=True, tree=False, seed=0,
                equal=False, magnitude=1.0):
    g = torch.Generator().manual_seed(seed)
    Bn, P = len(counts), len(members)
    lens = [max(0, rows - (7 * i) % 5 * (rows // 6)) if uneven else rows for i in range(Bn * layers * hk)]
    plens = [max(0, plen - (5 * i) % 4 * (plen // 5)) if uneven else plen for i in range(P * layers * hk)]
    buf = cache(Bn, rows, lens, dtype, D, hk, G, layers, g, max(counts) + 2, ragged=uneven, magnitude=magnitude)
    pre = cache(P, plen, plens, dtype, D, hk, G, layers, g, 5, ragged=uneven, magnitude=magnitude)
    tok = make_tokens(counts)
    q = torch.randn((sum(counts), hk * G, D), generator=g).to(TYPES[dtype]).cuda()
    parent = None
    if tree:
        r = np.random.default_rng(seed)
        parent = [int(r.integers(-1, i)) if i else -1 for _, _, n in spans(counts) for i in range(n)]
    sh = make_shared(pre, members[0] if equal else members)
    pt = None if parent is None else torch.tensor(parent, dtype=torch.int32, device="cuda")
    out = buf.shared_attention(tok, sh, q, pt, layer=layers - 1)
    torch.cuda.synchronize()
    check_shared(out, buf, pre, counts, members, lens, plens, q, dtype, parent, layers - 1)
    return buf, pre, tok, sh, q, pt, out, lens, plens


# ------------------------------------------------------------------------ shared rows

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_shared_small(dtype, D, tree):
    for i, (counts, members, plen, rows, hk, G, layers) in enumerate((
            ([1], [1], 1, 0, 1, 1, 1), ([1, 1, 1, 1], [4], 33, 2, 2, 2, 1), ([2, 0, 3, 1, 5], [2, 0, 2], 70, 40, 2, 4, 2),
            ([1] * 9, [3, 3, 3], 129, 0, 1, 8, 1), ([7, 20, 1], [1, 1], 200, 131, 3, 4, 1), ([33, 64], [2], 65, 17, 1, 8, 1))):
        print(f"shared {dtype} D={D} tree={tree} counts={counts} members={members}", flush=True)
        shared_case(counts, members, plen, rows, dtype, D, hk, G, layers, uneven=i % 2 == 0, tree=tree, seed=i)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("counts,members,plen,rows,G", [
    ([1] * 8, [8], 3001, 200, 4), ([1] * 20, [17, 2], 1500, 700, 4), ([3] * 16, [16], 2100, 50, 8),
    ([1, 90, 250], [2, 1], 900, 300, 2), ([1] * 40, [20, 20], 600, 1, 1)])
def test_shared_longer(dtype, D, counts, members, plen, rows, G):
    print(f"shared {dtype} D={D} counts={counts} plen={plen}", flush=True)
    shared_case(counts, members, plen, rows, dtype, D, 2, G, 1, seed=plen)


def test_shared_equal_groups_without_offsets():
    a = shared_case([2] * 6, [3, 3], 300, 20, uneven=False, equal=True, seed=4)
    b = shared_case([2] * 6, [3, 3], 300, 20, uneven=False, seed=4)
    assert not a[3].first and b[3].first and torch.equal(a[6], b[6])


def test_shared_many_workgroups():
    # past the size where streamed caches take tiles of 128 rows
    shared_case([1] * 12, [6, 6], 15000, 1500, hk=8, G=4, seed=8)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_shared_is_one_cache_in_two_pieces(dtype, D):
    buf, pre, tok, sh, q, _, out, _, _ = shared_case([1, 2, 30], [3], 400, 60, dtype, D, uneven=False, seed=2)
    both = cache(3, 460, None, dtype, D, 2, 4, 1, torch.Generator().manual_seed(0), 40, ragged=False)
    for u in range(6):
        both.k[u, :400], both.v[u, :400] = pre.k[u % 2, :400], pre.v[u % 2, :400]
        both.k[u, 400:490], both.v[u, 400:490] = buf.k[u, :90], buf.v[u, :90]
    whole = both.prompt_attention(tok, q)
    H = half_step(dtype)
    # each side is off as the header says; a weight is rounded against the maximum met so far, which differs
    off = 2 * (H * np.abs(np64(whole)) + ((500 + 8) * F + (2 * H if dtype == "bf16" else 0)) * float(both.v.abs().max()))
    assert np.all(np.abs(np64(out) - np64(whole)) <= off)


def test_shared_prefix_without_rows_is_the_prompt():
    buf, pre, tok, sh, q, _, _, lens, plens = shared_case([1, 4], [2], 50, 30, seed=5)
    pre.unit_len.zero_()
    want = buf.prompt_attention(tok, q)
    check_shared(buf.shared_attention(tok, sh, q), buf, pre, [1, 4], [2], lens, [0] * len(plens), q, "bf16")
    pre.kv.len = 0
    assert torch.equal(buf.shared_attention(tok, sh, q), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_shared_ignores_what_is_not_seen(dtype, D):
    for counts, members, plen, rows in (([1, 1, 1], [2], 90, 20), ([5, 40], [1, 1], 700, 300)):
        case = shared_case(counts, members, plen, rows, dtype, D, seed=9, tree=max(counts) > 1)
        buf, pre, tok, sh, q, pt, out, lens, plens = case
        parent = None if pt is None else pt.tolist()
        for bad in (float("nan"), float("inf")):
            for u, n in enumerate(plens):
                pre.k[u, n:], pre.v[u, n:] = bad, bad
            for u, n in enumerate(lens):
                m = counts[u // 2]
                buf.k[u, n + m:], buf.v[u, n + m:] = bad, bad
            # later tokens' value rows, and in a tree other branches': seen by some rows of a tile, not by others
            again = buf.shared_attention(tok, sh, q, pt)
            assert torch.isfinite(again).all()
            check_shared(again, buf, pre, counts, members, lens, plens, q, dtype, parent)
        u = 2 * (len(counts) - 1)
        buf.v[u, lens[u] + counts[-1] - 1] = float("inf")
        got = buf.shared_attention(tok, sh, q, pt)
        at = sum(counts[:-1])
        sees = mask_of(parent, at, counts[-1])[:, -1] if parent is not None else np.eye(counts[-1], dtype=bool)[-1]
        fin = torch.isfinite(got[at:, :4]).all(-1).all(-1).cpu().numpy()
        assert np.array_equal(fin, ~sees) and torch.isfinite(got[at:, 4:]).all() and torch.isfinite(got[:at]).all()


def test_shared_extremes_of_logits():
    # a lowest-value mask in the keys, large logits on one side only, and values near the largest number
    g = torch.Generator().manual_seed(1)
    for dtype in ("bf16", "f32"):
        buf, pre, tok, sh, q, _, _, lens, plens = shared_case([1, 3], [2], 260, 40, dtype, 64, seed=3, uneven=False)
        q.copy_(torch.sign(torch.randn(q.shape, generator=g)).to(q.dtype).cuda() * 8)
        pre.k[:, 7] = 40.0 * q[0, 0]
        pre.k[:, 100:140] = -300.0 * q[0, 0]
        out = buf.shared_attention(tok, sh, q)
        check_shared(out, buf, pre, [1, 3], [2], lens, plens, q, dtype)
        pre.v[:, 7] = 3e38
        buf.v[:, 5] = -3e38
        assert torch.isfinite(buf.shared_attention(tok, sh, q)).all()


def test_shared_padding_rows_are_left():
    buf, pre, _, sh, q, _, _, lens, plens = shared_case([2, 3, 1], [2, 1], 60, 10, seed=6)
    tok = make_tokens([2, 3, 1])
    cu = torch.tensor([3, 5, 8, 9], dtype=torch.int32, device="cuda")          # tokens 0..2 and 9.. are padding
    padded = B.dc_tokens(9, 3, cu.data_ptr())
    qq = torch.zeros((9,) + q.shape[1:], dtype=q.dtype, device="cuda")
    qq[3:9] = q
    out = torch.full_like(qq, 7.0)
    buf.shared_attention(padded, sh, qq, out=out)
    assert torch.equal(out[3:9], buf.shared_attention(tok, sh, q)) and (out[:3] == 7).all()


def test_shared_offsets_out_of_order_stay_in_the_buffers():
    buf, pre, tok, sh, q, _, out, _, _ = shared_case([2, 1, 3], [2, 1], 60, 10, seed=7)
    good = sh.first_tensor.clone()
    for bad in ([5, 2, 9], [-3, 1, 2], [0, 3, 1], [2, 2, 2], [2**31 - 1, -2**31, 1]):
        sh.first_tensor.copy_(torch.tensor(bad, dtype=torch.int32))
        buf.shared_attention(tok, sh, q)
    sh.first_tensor.copy_(good)
    assert torch.equal(buf.shared_attention(tok, sh, q), out)


# ------------------------------------------------------------------------ bounds

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [16, 32, 64, 128])
def test_bounds(dtype, D, rows):
    g = torch.Generator().manual_seed(rows + D)
    for batch, hk, layers, n, spare in ((1, 1, 1, rows, 0), (2, 2, 2, 5 * rows + 7, 3), (3, 1, 1, 41 * rows + 1, rows)):
        lens = [max(0, n - (3 * i) % 4 * (n // 3)) for i in range(batch * hk * layers)]
        buf = cache(batch, n, lens, dtype, D, hk, 2, layers, g, spare)
        buf.k[0, 1, 2], buf.k[0, 2, 3], buf.k[0, 3, 4] = float("inf"), float("-inf"), float("nan")
        buf.k[0, 4, 5] = -float("nan")
        buf.k[-1, :, 7] = -0.0
        blocks = buf.make_blocks(rows)
        blocks.bounds_tensor.fill_(9)
        buf.block_bounds(blocks)
        got, top = np64(blocks.bounds_tensor), float(torch.finfo(TYPES[dtype]).max)
        for u, m in enumerate(lens):
            k = np64(buf.k[u, :m])
            sign = torch.signbit(buf.k[u, :m]).cpu().numpy()
            k = np.where(np.isnan(k), np.where(sign, -top, top), k)
            assert np.array_equal(got[u, :m // rows], ob.bounds(k, rows, top)), (u, m)
            assert (got[u, m // rows:] == 9).all()


def test_bounds_from_a_row_on():
    g = torch.Generator().manual_seed(0)
    lens = [100, 64, 63, 31]
    buf = cache(2, 100, lens, g=g, spare=30)
    blocks = buf.make_blocks(16)
    buf.block_bounds(blocks)
    whole = blocks.bounds_tensor.clone()
    for start, redone in ((0, 0), (15, 0), (16, 1), (40, 2), (95, 5), (96, 6), (100, 6)):
        blocks.bounds_tensor.fill_(5)
        buf.block_bounds(blocks, start)
        for u, n in enumerate(lens):
            lo = min(redone, n // 16)
            assert (blocks.bounds_tensor[u, :lo] == 5).all()
            assert torch.equal(blocks.bounds_tensor[u, lo:n // 16], whole[u, lo:n // 16])
            assert (blocks.bounds_tensor[u, n // 16:] == 5).all()


# ------------------------------------------------------------------------ choice

def chosen_by_oracle(buf, bt, counts, q, rows, lens, count, share, first, last, layer):
    hk, G, L = buf.dims.n_kv_heads, buf.G, buf.dims.n_layers
    groups = -(-max(counts) // share)
    want = np.full((len(counts), groups, hk, count), -1)
    x, bd = np64(q), np64(bt)
    for b, at, n in spans(counts):
        for h in range(hk):
            u = (b * L + layer) * hk + h
            for i in range(-(-n // share)):
                qs = x[at + i * share:at + min((i + 1) * share, n), h * G:(h + 1) * G].reshape(-1, buf.D)
                want[b, i, h] = ob.choose(ob.scores(qs, bd[u, :lens[u] // rows]), count, first, last)
    return want


def select_case(counts, n, rows, count, share=1, first=0, last=0, dtype="bf16", D=128, hk=2, G=4, layers=1, seed=0):
    g = torch.Generator().manual_seed(seed)
    lens = [max(0, n - (3 * i) % 4 * (n // 5)) for i in range(len(counts) * hk * layers)]
    buf = cache(len(counts), n, lens, dtype, D, hk, G, layers, g, max(counts) + 1)
    blocks = buf.make_blocks(rows)
    buf.block_bounds(blocks)
    q = torch.randn((sum(counts), hk * G, D), generator=g).to(TYPES[dtype]).cuda()
    return buf, blocks, make_tokens(counts), q, lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_select(dtype, D):
    for i, (counts, n, rows, count, share, first, last, hk, G, layers) in enumerate((
            ([1], 40, 16, 1, 1, 0, 0, 1, 1, 1), ([1, 1, 1], 900, 16, 7, 1, 1, 2, 2, 4, 2), ([4, 0, 9], 700, 32, 5, 4, 0, 1, 2, 8, 1),
            ([3, 40], 1200, 16, 33, 16, 2, 0, 1, 2, 1), ([70, 3], 500, 64, 3, 50, 1, 1, 2, 4, 1), ([2], 15, 16, 4, 3, 1, 1, 2, 4, 1),
            ([1, 1], 3000, 128, 23, 1, 0, 0, 3, 4, 1), ([150], 400, 16, 24, 1000, 0, 0, 1, 8, 1))):
        print(f"select {dtype} D={D} counts={counts} n={n}", flush=True)
        buf, blocks, tok, q, lens = select_case(counts, n, rows, count, share, first, last, dtype, D, hk, G, layers, i)
        got = buf.block_select(tok, blocks, q, count, share, first, last, layer=layers - 1)
        want = chosen_by_oracle(buf, blocks.bounds_tensor, counts, q, rows, lens, count, share, first, last, layers - 1)
        assert np.array_equal(got.cpu().numpy(), want), i


@pytest.mark.parametrize("dtype,D,n,rows,count", [("bf16", 128, 20003, 16, 100), ("f32", 64, 16384 * 16, 16, 2048),
                                                 ("bf16", 64, 70001, 32, 1500), ("bf16", 128, 16384 * 16, 16, 7)])
def test_select_of_many_blocks(dtype, D, n, rows, count):
    buf, blocks, tok, q, lens = select_case([1], n, rows, count, dtype=dtype, D=D, hk=2, G=2)
    got = buf.block_select(tok, blocks, q, count, first=1, last=2)
    want = chosen_by_oracle(buf, blocks.bounds_tensor, [1], q, rows, lens, count, 1, 1, 2, 0)
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("blocks", [5, 64, 255, 256, 257, 511, 512, 513, 1023, 1024, 1025, 2049, 4097])
def test_select_at_the_sizes_where_the_search_changes(blocks):
    n = 16 * blocks + 3
    for batch, counts in ((1, (1, 4)), (40, (4,))):       # few lists, and more than half the CUs' number of heads
        if batch * blocks > 42000:
            continue
        buf, bl, tok, q, lens = select_case([1] * batch, n, 16, 0, D=64, hk=8 if batch > 1 else 2, G=2, seed=blocks)
        for count in counts + (blocks - 1, blocks):
            if count > 2048 or batch > 1 and count > 4:
                continue
            for first, last in ((0, 0), (1, 3), (count, 0), (0, count), (min(2, count), 0)):   # (all of them forced, too)
                if first + last > count:
                    continue
                got = buf.block_select(tok, bl, q, count, first=first, last=last)
                want = chosen_by_oracle(buf, bl.bounds_tensor, [1] * batch, q, 16, lens, count, 1, first, last, 0)
                assert np.array_equal(got.cpu().numpy(), want), (batch, count, first, last)
        # seven kinds of blocks, so that the limit falls among equals; then all equal
        x, count = bl.bounds_tensor, min(blocks, 2048) // 2 + 1
        x.copy_(x[:, torch.arange(x.shape[1], device="cuda") % 7])
        for _ in range(2):
            got = buf.block_select(tok, bl, q, count, first=1)
            want = chosen_by_oracle(buf, x, [1] * batch, q, 16, lens, count, 1, 1, 0, 0)
            assert np.array_equal(got.cpu().numpy(), want), (batch, count)
            q.zero_()


def test_select_ties_and_values_that_are_no_numbers():
    buf, blocks, tok, q, lens = select_case([1, 1, 1], 600, 16, 9, hk=1, G=4, seed=3)
    # equal blocks: the lower numbers, by threes
    x = blocks.bounds_tensor
    x[:, :36] = x[:, :12].repeat_interleave(3, 1)
    for count in (1, 2, 3, 4, 10, 11, 20):
        got = buf.block_select(tok, blocks, q, count).cpu().numpy()
        assert np.array_equal(got, chosen_by_oracle(buf, x, [1] * 3, q, 16, lens, count, 1, 0, 0, 0)), count
    q[0] = 0                                              # all scores equal
    q[1, 0, 5] = float("nan")                             # and none a number
    q[2, 2, 7] = float("inf")
    got = buf.block_select(tok, blocks, q, 5, first=0, last=1).cpu()
    for b in (0, 1):
        assert got[b, 0, 0].tolist() == [0, 1, 2, 3, lens[b] // 16 - 1]
    assert len(set(got[2, 0, 0].tolist())) == 5 and got.min() >= 0
    # a block that holds NaN or infinite keys has finite bounds, and is chosen rather than passed over
    buf.k[0, 77, 3] = float("nan")
    buf.block_bounds(blocks)
    q[0] = 1.0
    assert 77 // 16 in buf.block_select(tok, blocks, q, 3)[0, 0, 0].tolist()


# ------------------------------------------------------------------------ attention over chosen blocks

def check_blocks(out, buf, counts, lens, lists, q, rows, share, dtype, layer=0):
    hk, G, L = buf.dims.n_kv_heads, buf.G, buf.dims.n_layers
    o, x, ls = np64(out), np64(q), lists.cpu().numpy()
    for b, at, n in spans(counts):
        for h in range(hk):
            u = (b * L + layer) * hk + h
            K, V = np64(buf.k[u]), np64(buf.v[u])
            for i in range(-(-n // share)):
                t0, t1 = i * share, min((i + 1) * share, n)
                at_rows = ob.rows_of(ls[b, i, h], rows, lens[u])
                old = len(at_rows)
                at_rows = at_rows + list(range(lens[u], lens[u] + t1))
                see = np.arange(len(at_rows))[None] <= old + np.arange(t0, t1)[:, None]
                bad = attention_off(o[at + t0:at + t1, h * G:(h + 1) * G], x[at + t0:at + t1, h * G:(h + 1) * G],
                                    K[at_rows], V[at_rows], see, dtype)
                assert not bad, (b, h, i, bad)


def lists_for(counts, lens, rows, count, share, hk, layers, layer, seed, rough=False):
    r = np.random.default_rng(seed)
    out = np.full((len(counts), -(-max(counts) // share), hk, count), -1)
    for b in range(len(counts)):
        for i in range(out.shape[1]):
            for h in range(hk):
                c = lens[(b * layers + layer) * hk + h] // rows
                if rough:
                    out[b, i, h] = r.integers(-3, c + 3, count)       # unordered, repeated, outside
                else:
                    k = min(c, int(r.integers(0, count + 1)))
                    out[b, i, h, :k] = np.sort(r.permutation(c)[:k])
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def blocks_case(counts, n, rows, count, share, dtype="bf16", D=128, hk=2, G=4, layers=1, seed=0, rough=False, uneven=True):
    g = torch.Generator().manual_seed(seed)
    lens = [max(0, n - (3 * i) % 4 * (n // 5)) if uneven else n for i in range(len(counts) * hk * layers)]
    buf = cache(len(counts), n, lens, dtype, D, hk, G, layers, g, max(counts) + 1, ragged=uneven)
    blocks, tok = buf.make_blocks(rows), make_tokens(counts)
    q = torch.randn((sum(counts), hk * G, D), generator=g).to(TYPES[dtype]).cuda()
    lists = lists_for(counts, lens, rows, count, share, hk, layers, layers - 1, seed, rough)
    out = buf.block_attention(tok, blocks, lists, q, share, layer=layers - 1)
    torch.cuda.synchronize()
    check_blocks(out, buf, counts, lens, lists, q, rows, share, dtype, layers - 1)
    return buf, blocks, tok, q, lens, lists, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rough", [False, True])
def test_block_attention(dtype, D, rough):
    for i, (counts, n, rows, count, share, hk, G, layers) in enumerate((
            ([1], 0, 16, 1, 1, 1, 1, 1), ([1], 16, 16, 1, 1, 1, 1, 1), ([1, 1, 1], 500, 16, 9, 1, 2, 4, 2),
            ([3, 0, 17], 700, 32, 8, 4, 2, 2, 1), ([5, 70], 900, 64, 6, 32, 1, 8, 1), ([130], 600, 128, 3, 40, 2, 4, 1),
            ([2, 2], 900, 16, 50, 2, 2, 8, 1), ([40], 1000, 16, 70, 64, 1, 2, 1))):
        print(f"blocks {dtype} D={D} rough={rough} counts={counts} n={n}", flush=True)
        blocks_case(counts, n, rows, count, share, dtype, D, hk, G, layers, i, rough)


@pytest.mark.parametrize("dtype,D,counts,n,rows,count,share,G", [
    ("bf16", 128, [1] * 4, 9000, 64, 60, 1, 4), ("bf16", 64, [1], 30000, 16, 1000, 1, 8), ("f32", 128, [1, 1], 5000, 32, 64, 1, 2),
    ("f32", 64, [100], 3000, 16, 90, 64, 4), ("bf16", 128, [300], 4000, 64, 20, 32, 4), ("bf16", 128, [1], 40000, 16, 2048, 1, 1)])
def test_block_attention_longer(dtype, D, counts, n, rows, count, share, G):
    blocks_case(counts, n, rows, count, share, dtype, D, 2, G, seed=n, uneven=n != 9000)


def test_block_attention_over_a_large_batch():
    # past the size where streamed rows take tiles of 128
    blocks_case([1] * 32, 2600, 64, 34, 1, hk=4, G=4, seed=1, uneven=False)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_all_blocks_are_the_whole_cache(dtype, D):
    buf, blocks, tok, q, lens, _, _ = blocks_case([3, 1], 300, 16, 20, 2, dtype, D, seed=4)
    buf.block_bounds(blocks)
    out = buf.sparse_attention(tok, blocks, q, 20, share=2)
    whole = buf.prompt_attention(tok, q)
    H = half_step(dtype)
    off = 2 * (H * np.abs(np64(whole)) + ((304 + 8) * F + (2 * H if dtype == "bf16" else 0)) * float(buf.v.abs().max()))
    assert np.all(np.abs(np64(out) - np64(whole)) <= off)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_blocks_that_are_not_chosen_have_no_influence(dtype, D):
    for counts, n, share in (([1, 1], 400, 1), ([30], 500, 8)):
        buf, blocks, tok, q, lens, lists, out = blocks_case(counts, n, 16, 6, share, dtype, D, seed=11)
        for bad in (float("nan"), float("inf")):
            for u, m in enumerate(lens):
                b, h = divmod(u, 2)
                used = {r for i in range(lists.shape[1]) for r in ob.rows_of(lists[b, i, h].cpu().numpy(), 16, m)}
                free = [r for r in range(m) if r not in used] + list(range(m + counts[b], buf.cap))
                buf.k[u, free], buf.v[u, free] = bad, bad
            assert torch.equal(buf.block_attention(tok, blocks, lists, q, share), out)
        # a value row of the last token: infinite only for those who see it
        buf.v[0, lens[0] + counts[0] - 1] = float("inf")
        got = torch.isfinite(buf.block_attention(tok, blocks, lists, q, share)[:counts[0], :4]).all(-1).all(-1)
        assert got[:-1].all() and not got[-1]


def test_block_attention_leaves_padding():
    buf, blocks, tok, q, lens, lists, out = blocks_case([2, 3], 200, 16, 4, 2, seed=5)
    cu = torch.tensor([1, 3, 6], dtype=torch.int32, device="cuda")
    padded = B.dc_tokens(6, 3, cu.data_ptr())
    qq = torch.zeros((6,) + q.shape[1:], dtype=q.dtype, device="cuda")
    qq[1:] = q
    o = torch.full_like(qq, 7.0)
    buf.block_attention(padded, blocks, lists, qq, 2, out=o)
    assert torch.equal(o[1:], out) and (o[0] == 7).all()
    buf.block_bounds(blocks)
    assert torch.equal(buf.block_select(padded, blocks, qq, 4, 2), buf.block_select(tok, blocks, q, 4, 2))


def test_rows_past_32_bits():
    # one unit of 2^24 + 300 rows of 128 bf16: bytes past 2^32, elements past 2^31
    n, D = (1 << 24) + 300, 128
    buf = DecodeBuffers(1, 1, 4, 1, D, n + 2, "bf16", features=False)
    g = torch.Generator().manual_seed(0)
    buf.kv.len = n
    far = torch.randn((400, D), generator=g).to(torch.bfloat16).cuda()
    buf.k[0, n - 399:n + 1], buf.v[0, n - 399:n + 1] = far, far.flip(0)
    blocks = buf.make_blocks(128)
    q = torch.randn((1, 4, D), generator=g).to(torch.bfloat16).cuda()
    last = n // 128 - 1
    buf.block_bounds(blocks, n - 300)
    got = np64(blocks.bounds_tensor[0, last - 1:last + 1])
    assert np.array_equal(got, ob.bounds(np64(buf.k[0, (last - 1) * 128:(last + 1) * 128]), 128, 3e38))
    lists = torch.tensor([[[[last - 1, last]]]], dtype=torch.int32, device="cuda")
    out = buf.block_attention(make_tokens([1]), blocks, lists, q)
    rows = list(range((last - 1) * 128, n + 1))
    K, V = np64(buf.k[0, rows]), np64(buf.v[0, rows])
    assert not attention_off(np64(out), np64(q), K, V, np.ones((1, len(rows)), bool), "bf16")
    # the same rows as a prefix of another cache
    own = cache(1, 5, None, hk=1, g=g, ragged=False)
    pre_rows = n
    pre = DecodeBuffers(1, 1, 4, 1, D, 8, "bf16", features=False)
    pre.k, pre.v, pre.cap = buf.k, buf.v, buf.cap
    pre.dims.capacity, pre.kv.k, pre.kv.v, pre.kv.len = buf.cap, buf.kv.k, buf.kv.v, pre_rows
    out = own.shared_attention(make_tokens([1]), make_shared(pre, 1), q)
    # most of the prefix are zero rows: their logit is 0, their value 0
    x = 1 / np.sqrt(D) * np64(q)[0] @ np64(far[:399]).T
    y = 1 / np.sqrt(D) * np64(q)[0] @ np64(own.k[0, :6]).T
    e, f = np.exp(x), np.exp(y)
    total = e.sum(1) + f.sum(1) + (n - 399)
    ref = (e @ np64(buf.v[0, n - 399:n]) + f @ np64(own.v[0, :6])) / total[:, None]
    mass = (e @ np.abs(np64(buf.v[0, n - 399:n])) + f @ np.abs(np64(own.v[0, :6]))) / total[:, None]
    # the sum of 2^24 weights: ones, added in float32 within a lane's share of a part and then over parts; a
    # sum of k equal terms is off by k F at most, k = rows of a part / 32 lanes' halves + the parts
    H = half_step("bf16")
    k = n // 64 / 2 + 64
    assert np.all(np.abs(np64(out)[0] - ref) <= 2 * H * np.abs(ref) + (k * F + 3 * H) * mass)


# ------------------------------------------------------------------------ together

def test_run_together():
    """Two prompts prefilled as prefixes; five rollouts take steps over them; and one cache that grows past its blocks,
    part by part and then token by token, read sparsely."""
    g = torch.Generator().manual_seed(3)
    hk, G, D, td = 2, 4, 128, torch.bfloat16
    rope = make_rope(10000.0 ** (-torch.arange(64, device="cuda") / 64), norm=True)

    def parts(n):
        x = torch.randn((n, (hk * G + 2 * hk) * D), generator=g).to(td).cuda().unflatten(1, (hk * G + 2 * hk, D))
        return x[:, :hk * G], x[:, hk * G:hk * G + hk], x[:, hk * G + hk:]

    def pos(starts, counts):
        return torch.cat([torch.arange(s, s + n, dtype=torch.int32) for s, n in zip(starts, counts)]).cuda()

    counts = [150, 60]
    pre = DecodeBuffers(2, 1, hk * G, hk, D, 200, ragged=True, features=False)
    tok = make_tokens(counts)
    pre.prefill(tok, rope, *parts(210), pos([0, 0], counts))
    pre.commit_rows(tok)
    rolls = DecodeBuffers(5, 1, hk * G, hk, D, 40, features=False)
    sh, one = make_shared(pre, [3, 2]), make_tokens([1] * 5)
    base = [150] * 3 + [60] * 2
    for step in range(4):
        q, k, v = parts(5)
        q, _ = rolls.norm_rope(one, rope, q, k, v, pos([b + step for b in base], [1] * 5))
        out = rolls.shared_attention(one, sh, q)
        plens = pre.unit_len.tolist()
        check_shared(out, rolls, pre, [1] * 5, [3, 2], [step] * 10, plens, q, "bf16")
        rolls.commit_rows(one)
    assert rolls.len == 4

    buf = DecodeBuffers(1, 1, hk * G, hk, D, 400, features=False)
    blocks, at = buf.make_blocks(16), 0
    for n, share in ((100, 25), (90, 30), (50, 25), (1, 1), (1, 1), (1, 1)):
        tok = make_tokens([n])
        q, k, v = parts(n)
        q, _ = buf.norm_rope(tok, rope, q, k, v, pos([at], [n]))
        chosen = buf.block_select(tok, blocks, q, 4, share, first=1, last=1)
        want = chosen_by_oracle(buf, blocks.bounds_tensor, [n], q, 16, [at] * hk, 4, share, 1, 1, 0)
        assert np.array_equal(chosen.cpu().numpy(), want)
        out = buf.block_attention(tok, blocks, chosen, q, share)
        check_blocks(out, buf, [n], [at] * hk, chosen, q, 16, share, "bf16")
        assert torch.equal(out, buf.sparse_attention(tok, blocks, q, 4, share, 1, 1))
        buf.commit_rows(tok)
        buf.block_bounds(blocks, at)
        at += n


def test_graph_replays_and_other_streams():
    buf, pre, tok, sh, q, _, _, lens, plens = shared_case([1] * 6, [4, 2], 700, 90, seed=12)
    big, blocks, one, qb, blens, _, _ = blocks_case([1] * 3, 900, 16, 8, 1, seed=12)
    big.block_bounds(blocks)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    want = buf.shared_attention(tok, sh, q), big.sparse_attention(one, blocks, qb, 8)
    with torch.cuda.stream(s):
        for _ in range(2):
            buf.shared_attention(tok, sh, q)
            big.sparse_attention(one, blocks, qb, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a = buf.shared_attention(tok, sh, q)
        big.block_bounds(blocks)
        c = big.sparse_attention(one, blocks, qb, 8)
    for i in range(3):
        a.zero_()
        c.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(c, want[1])
        q.mul_(-1.0)                                 # the same graph over other inputs
        qb.mul_(-1.0)
        big.k.mul_(0.5)
        big.block_bounds(blocks)
        want = buf.shared_attention(tok, sh, q), big.sparse_attention(one, blocks, qb, 8)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    x = buf.shared_attention(tok, sh, q, stream=other)
    other.synchronize()
    y = big.sparse_attention(one, blocks, qb, 8, stream=other)
    other.synchronize()
    assert torch.equal(x, want[0]) and torch.equal(y, want[1])


def test_calls_are_repeatable_and_buffers_refuse():
    buf, pre, tok, sh, q, _, out, _, _ = shared_case([1] * 6, [4, 2], 2000, 90, seed=13)
    for _ in range(3):
        assert torch.equal(buf.shared_attention(tok, sh, q), out)
    with pytest.raises(ValueError):
        buf.shared_attention(tok, sh, q.float())
    with pytest.raises(ValueError):
        buf.shared_attention(make_tokens([1] * 5), sh, q[:5])
    other = cache(6, 20, None, hk=4, G=2, ragged=False)
    with pytest.raises(ValueError):
        other.shared_attention(tok, sh, q)
    with pytest.raises(ValueError):
        make_shared(pre, [4])
    with pytest.raises(ValueError):
        make_shared(pre, [4, -1])
    blocks = buf.make_blocks(16)
    with pytest.raises(ValueError):
        other.block_bounds(blocks)
    with pytest.raises(ValueError):
        buf.make_blocks(20)
    with pytest.raises(ValueError):
        buf.block_select(tok, blocks, q, 0)
    with pytest.raises(B.DCError):
        buf.block_select(tok, blocks, q, 2, first=2, last=1)
    with pytest.raises(ValueError):
        buf.block_attention(tok, blocks, torch.zeros((6, 1, 2, 3), device="cuda"), q)
    with pytest.raises(ValueError):
        buf.block_attention(tok, blocks, torch.zeros((6, 2, 2, 3), dtype=torch.int32, device="cuda"), q)


def test_blocks_of_a_cache_that_decodes_and_evicts():
    """Decode steps append rows and evictions move them: the bounds follow, and the blocks are those of the slots."""
    from paper_2608_08878_amd.buffers import make_policy
    g = torch.Generator().manual_seed(4)
    buf = DecodeBuffers(2, 1, 8, 2, 128, 200)
    buf.k.copy_(torch.randn(buf.k.shape, generator=g))
    buf.v.copy_(torch.randn(buf.v.shape, generator=g))
    buf.feat_init(150)
    pol = make_policy((0.3 * torch.randn(4 * 32 + 32 + 32 + 1, generator=g)).cuda(), (32,))
    blocks = buf.make_blocks(16)
    buf.block_bounds(blocks)

    def holds():
        n, bd = buf.len // 16, np64(blocks.bounds_tensor)
        return all(np.array_equal(bd[u, :n], ob.bounds(np64(buf.k[u, :buf.len]), 16, 3e38)) for u in range(4))

    def heads(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16).cuda()

    assert holds()
    for _ in range(20):
        before = buf.len
        buf.decode_step(heads(4, 4, 128), heads(4, 128), heads(4, 128))
        buf.block_bounds(blocks, before)
        assert holds()
    buf.decode_evict(pol, 90, heads(4, 4, 128), heads(4, 128), heads(4, 128))
    assert buf.len == 90
    buf.block_bounds(blocks)
    assert holds()
    tok, q = make_tokens([1, 1]), heads(2, 8, 128)
    lists = buf.block_select(tok, blocks, q, 3)
    out = buf.block_attention(tok, blocks, lists, q)
    check_blocks(out, buf, [1, 1], [90] * 4, lists, q, 16, 1, "bf16")
    buf.shrink(100)
    with pytest.raises(ValueError):
        buf.block_bounds(blocks)
    again = buf.make_blocks(16)
    buf.block_bounds(again)
    assert torch.equal(again.bounds_tensor[:, :5], blocks.bounds_tensor[:, :5])


def test_shared_rows_of_several_layers_and_shrunken_prefixes():
    buf, pre, tok, sh, q, _, out, lens, plens = shared_case([1, 2, 1], [2, 1], 90, 20, layers=3, seed=21)
    pre.shrink(92)
    assert torch.equal(buf.shared_attention(tok, sh, q, layer=2), out)
    for layer in range(3):
        check_shared(buf.shared_attention(tok, sh, q, layer=layer), buf, pre, [1, 2, 1], [2, 1], lens, plens, q, "bf16",
                     layer=layer)


def test_workspaces_that_a_call_outgrows_stay_for_graphs():
    buf, pre, tok, sh, q, _, out, _, _ = shared_case([1, 1], [2], 300, 20, seed=22)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured = buf.shared_attention(tok, sh, q)
    old = buf.ws_bytes
    buf._grow(64 * old)                                  # as a later, larger call would
    torch.full((old // 4,), float("nan"), device="cuda")
    for _ in range(3):
        captured.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, want)
        assert torch.equal(buf.shared_attention(tok, sh, q), want)
