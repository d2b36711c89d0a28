"""Device buffers for the C-ABI structs, allocated with torch (device memory and
streams only; no computation happens here)."""
from __future__ import annotations

import ctypes

import torch

from . import binding as B

TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
DC_DTYPE = {"f32": B.DC_F32, "bf16": B.DC_BF16}


def stream_handle(stream=None):
    if stream is None:
        # the raw handle: building a Stream object costs 2.8 us of a small call
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


class DecodeBuffers:
    """K/V cache and (optionally) feature state for `units` caches of `capacity` rows."""

    def __init__(self, batch, n_layers, n_q_heads, n_kv_heads, head_dim, capacity, dtype="bf16",
                 ent_window=64, scale=0.0, features=True, device="cuda", sigma=False,
                 ragged=False, alpha_recent=False):
        self.G = n_q_heads // n_kv_heads
        self.U = batch * n_layers * n_kv_heads
        self.D = head_dim
        self.cap = capacity
        self.dtype = dtype
        self.window = ent_window
        td = TORCH_DTYPE[dtype]
        self.dims = B.dc_dims(batch, n_layers, n_q_heads, n_kv_heads, head_dim, capacity,
                              DC_DTYPE[dtype], ent_window, scale)
        self.k = torch.zeros((self.U, capacity, head_dim), dtype=td, device=device)
        self.v = torch.zeros((self.U, capacity, head_dim), dtype=td, device=device)
        self.kv = B.dc_kv(self.k.data_ptr(), self.v.data_ptr(), 0)
        self.unit_len = None
        if ragged:
            # per-unit lengths on the device (units may keep different row counts)
            self.unit_len = torch.zeros(self.U, dtype=torch.int32, device=device)
            self.kv.unit_len = self.unit_len.data_ptr()
        self.feat = None
        if features:
            self.alpha = torch.zeros((self.U, capacity), dtype=torch.float32, device=device)
            self.num = torch.zeros((self.U, capacity), dtype=torch.float64, device=device)
            self.den = torch.zeros((self.U, capacity), dtype=torch.float64, device=device)
            self.pos = torch.zeros((self.U, capacity), dtype=torch.int32, device=device)
            self.vnorm = torch.zeros((self.U, capacity), dtype=torch.float32, device=device)
            w = max(ent_window, 1)
            self.qring = torch.zeros((self.U, w, self.G, head_dim), dtype=td, device=device)
            self.qstat = torch.zeros((self.U, w, self.G, 3), dtype=torch.float32, device=device)
            self.feat = B.dc_feat(self.alpha.data_ptr(), self.num.data_ptr(), self.den.data_ptr(),
                                  self.pos.data_ptr(), self.vnorm.data_ptr(),
                                  self.qring.data_ptr(), self.qstat.data_ptr(), 0, 0)
            self.feat.alpha_recent = int(alpha_recent)
            self.ga_ws = None
            self.sigma = None
            if sigma:
                # the fifth feature (needed by five-input policies)
                self.sigma = torch.zeros((self.U, capacity), dtype=torch.float32, device=device)
                self.feat.sigma = self.sigma.data_ptr()
            if ragged:
                # sequences that see different numbers of tokens
                self.behind = torch.zeros((B.BEHIND_ROWS, self.U), dtype=torch.int32, device=device)
                self.feat.behind = self.behind.data_ptr()
        self.ws = None
        self.ws_bytes = 0
        self._older_ws = []
        self._device = self.k.get_device()
        if features:
            self.reserve_workspace(capacity)

    @property
    def len(self) -> int:
        return self.kv.len

    def shrink(self, capacity: int):
        """Move the valid rows of every unit into buffers of a smaller capacity (device
        copies; the old buffers are released).  After a compression step only
        budget + 1 rows per unit are ever live, and the steady steps stream fewer
        distinct pages when each unit's rows sit closer together."""
        n = self.kv.len
        if capacity < n + 1:
            raise ValueError(f"capacity {capacity} cannot hold {n} rows plus an append")
        td = self.k.dtype
        dev = self.k.device

        def moved(t):
            out = torch.zeros((t.shape[0], capacity) + tuple(t.shape[2:]), dtype=t.dtype, device=dev)
            out[:, :n] = t[:, :n]
            return out

        self.k = moved(self.k)
        self.v = moved(self.v)
        self.kv.k, self.kv.v = self.k.data_ptr(), self.v.data_ptr()
        if self.feat is not None:
            self.alpha, self.num, self.den = moved(self.alpha), moved(self.num), moved(self.den)
            self.pos, self.vnorm = moved(self.pos), moved(self.vnorm)
            if self.sigma is not None:
                self.sigma = moved(self.sigma)
                self.feat.sigma = self.sigma.data_ptr()
            self.feat.alpha, self.feat.ent_num = self.alpha.data_ptr(), self.num.data_ptr()
            self.feat.ent_den, self.feat.pos = self.den.data_ptr(), self.pos.data_ptr()
            self.feat.vnorm = self.vnorm.data_ptr()
        self.cap = capacity
        self.dims.capacity = capacity
        assert self.k.dtype == td
        torch.cuda.synchronize(dev)

    def reserve_workspace(self, max_len: int, kl_rows: int = 0, kl_vocab: int = 0):
        self._grow(B.dc_workspace_bytes(self.dims, max_len, kl_rows, kl_vocab))
        return self.ws

    def _grow(self, need: int, stream=None):
        """A workspace of at least `need` bytes.  A captured graph may hold an outgrown one's
        address, so those live as long as the buffers; each is at least twice the one before,
        so that they add up to less than the present one."""
        if need <= self.ws_bytes:
            return
        if self.ws is not None:
            self._older_ws.append(self.ws)
            need = max(need, 2 * self.ws_bytes)
        need = -(-need // 16) * 16
        self.ws = self._empty((need // self.k.element_size(),), stream).view(torch.uint8)
        self.ws_bytes = need

    def feat_init(self, length: int, first_pos: int = 0, stream=None):
        self.kv.len = length
        if self.unit_len is not None:
            self.unit_len.fill_(length)
        B.dc_feat_init(self.dims, self.kv, self.feat, first_pos, stream_handle(stream))

    def decode_step(self, q, k_new=None, v_new=None, out=None, stream=None, features=True):
        if out is None:
            out = torch.empty_like(q)
        B.dc_decode_step(self.dims, self.kv, self.feat if features else None, q, k_new, v_new,
                         out, self.ws, self.ws_bytes, stream_handle(stream))
        return out

    def decode_evict(self, policy, budget, q, k_new=None, v_new=None, out=None, scores_out=None,
                     kept_out=None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        B.dc_decode_evict(self.dims, self.kv, self.feat, policy, budget, q, k_new, v_new, out,
                          scores_out, kept_out, self.ws, self.ws_bytes, stream_handle(stream))
        return out

    def global_alpha(self, stream=None):
        """Replace every row's recent alpha by its average over the sequence's
        units (all layers and KV heads) at the row's position."""
        need = B.dc_global_alpha_workspace_bytes(self.dims, self.feat.next_pos)
        if self.ga_ws is None or self.ga_ws.numel() < need:
            self.ga_ws = torch.empty(need, dtype=torch.uint8, device=self.k.device)
        B.dc_global_alpha(self.dims, self.kv, self.feat, self.ga_ws, self.ga_ws.numel(),
                          stream_handle(stream))

    def score_evict(self, policy, budget, scores_out=None, kept_out=None, stream=None):
        B.dc_score_evict(self.dims, self.kv, self.feat, policy, budget, scores_out, kept_out,
                         self.ws, self.ws_bytes, stream_handle(stream))


    def decode_sample_evict(self, policy, budget, gumbel, q, k_new=None, v_new=None, out=None,
                            scores_out=None, kept_out=None, logp_out=None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        B.dc_decode_sample_evict(self.dims, self.kv, self.feat, policy, budget, gumbel, q, k_new,
                                 v_new, out, scores_out, kept_out, logp_out, self.ws, self.ws_bytes,
                                 stream_handle(stream))
        return out

    def decode_evict_units(self, policy, budgets, max_budget, q, k_new, v_new, out=None,
                           scores_out=None, kept_out=None, stream=None):
        """One decode step of a ragged cache with per-unit budgets (decode, then the
        deterministic per-unit selection); units that fit on chip run it in one launch."""
        if out is None:
            out = torch.empty_like(q)
        B.dc_decode_evict_units(self.dims, self.kv, self.feat, policy, budgets, max_budget, q,
                                k_new, v_new, out, scores_out, kept_out, self.ws, self.ws_bytes,
                                stream_handle(stream))
        return out

    def score_evict_units(self, policy, budgets, max_budget, gumbel=None, scores_out=None,
                          kept_out=None, logp_out=None, stream=None):
        B.dc_score_evict_units(self.dims, self.kv, self.feat, policy, budgets, max_budget, gumbel,
                               scores_out, kept_out, logp_out, self.ws, self.ws_bytes,
                               stream_handle(stream))

    def sample_evict(self, policy, budget, gumbel, scores_out=None, kept_out=None, logp_out=None,
                     stream=None):
        B.dc_sample_evict(self.dims, self.kv, self.feat, policy, budget, gumbel, scores_out,
                          kept_out, logp_out, self.ws, self.ws_bytes, stream_handle(stream))


    # ---- several tokens at once: prompts and drafted tokens

    # (the checks cost host time on calls of a few microseconds: plain comparisons)

    def _rows_of(self, x, heads, tokens, name):
        """x [N][heads][d] with dense rows: its elements from token to token."""
        n, d = tokens.tokens, self.D
        if x.dtype != self.k.dtype or x.shape != (n, heads, d):
            raise ValueError(f"{name} must be {self.k.dtype} [{n}][{heads}][{d}], got {x.dtype} {list(x.shape)}")
        ld, between, one = x.stride()
        if one != 1 or (between != d and heads > 1):
            raise ValueError(f"{name}'s heads must be contiguous within a token")
        self._here(x, name)
        return ld if n > 1 else heads * d        # (a single token's stride is never used)

    def _like(self, x, tokens, heads, name):
        """An output given by the caller."""
        if self._rows_of(x, heads, tokens, name) != heads * self.D:
            raise ValueError(f"{name} must be contiguous")
        return x

    def _ints(self, x, shape, name):
        if x.dtype != torch.int32 or x.shape != shape or not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous int32 {list(shape)}, got {x.dtype} {list(x.shape)}")
        self._here(x, name)

    def _batch_of(self, tokens):
        n = getattr(tokens, "sequences", self.dims.batch)
        if n != self.dims.batch:
            raise ValueError(f"tokens of {n} sequences for a cache of {self.dims.batch}")
        if getattr(tokens, "device", self._device) != self._device:
            raise ValueError(f"the tokens' offsets are on cuda:{tokens.device}, the cache on {self.k.device}")

    def _rope_of(self, rope):
        """What make_rope noted of its vectors, against this cache."""
        if getattr(rope, "gain_len", self.D) != self.D:
            raise ValueError(f"gains of {rope.gain_len} elements for heads of {self.D}")
        if getattr(rope, "device", self._device) != self._device:
            raise ValueError(f"the rotation's vectors are on cuda:{rope.device}, the cache on {self.k.device}")

    def _here(self, x, name):
        if x.get_device() != self._device:
            raise ValueError(f"{name} is on {x.device}, the cache on {self.k.device}")

    def _stream_here(self, stream):
        """The stream's handle; the cache has to be on the current device, which launches it."""
        here = torch.cuda.current_device()
        if here != self._device:
            raise ValueError(f"the cache is on {self.k.device}, the current device is cuda:{here}")
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(here)) if stream is None else stream_handle(stream)

    def _empty(self, shape, stream):
        """A tensor of the cache's type in memory that the given stream uses first (the allocator
        orders reuse by stream)."""
        if stream is None:
            return self.k.new_empty(shape)
        with torch.cuda.stream(stream):
            return self.k.new_empty(shape)

    def norm_rope(self, tokens, rope, q, k, v=None, pos=None, layer=0, q_out=None, k_out=None, stream=None):
        """Queries and keys of `tokens` normed and rotated (dc_qk_norm_rope).  With v the rotated
        keys and the values go into the cache behind its rows; without, the keys are
        returned too.  Returns (q_out, k_out or None)."""
        hq, hk = self.dims.n_q_heads, self.dims.n_kv_heads
        self._batch_of(tokens)
        self._rope_of(rope)
        ld_q, ld_k = self._rows_of(q, hq, tokens, "q"), self._rows_of(k, hk, tokens, "k")
        if pos is not None:
            self._ints(pos, (tokens.tokens,), "pos")
        q_out = self._empty(q.shape, stream) if q_out is None else self._like(q_out, tokens, hq, "q_out")
        ld_v = 0
        if v is not None:
            if k_out is not None:
                raise ValueError("with v the keys go to the cache: no k_out")
            ld_v = self._rows_of(v, hk, tokens, "v")
        else:
            k_out = self._empty(k.shape, stream) if k_out is None else self._like(k_out, tokens, hk, "k_out")
        B.dc_qk_norm_rope(self.dims, self.kv, layer, tokens, rope, q, ld_q, k, ld_k, v, ld_v, pos, q_out, k_out,
                          self._stream_here(stream))
        return q_out, k_out

    def reserve_tokens_workspace(self, tokens, max_len: int, stream=None):
        """Scratch of the attention of such tokens over caches of up to max_len rows, the tokens' own
        included.  The calls reserve what they need themselves; reserved once for the longest cache,
        it does not grow on the way.  All calls of one DecodeBuffers share it: they, and replays of
        graphs that captured them, run one after the other."""
        self._grow(B.dc_tokens_workspace_bytes(self.dims, tokens, max_len), stream)

    def _check_queries(self, tokens, q, out, stream):
        self._batch_of(tokens)
        hq = self.dims.n_q_heads
        self._like(q, tokens, hq, "q")
        return self._empty(q.shape, stream) if out is None else self._like(out, tokens, hq, "out")

    def prompt_attention(self, tokens, q, layer=0, out=None, stream=None):
        """Causal attention of packed prompts whose K/V are behind the cache's rows."""
        out = self._check_queries(tokens, q, out, stream)
        self.reserve_tokens_workspace(tokens, self.kv.len + tokens.max_tokens, stream)
        B.dc_prompt_attention(self.dims, self.kv, layer, tokens, q, out, self.ws, self.ws_bytes,
                              self._stream_here(stream))
        return out

    def tree_attention(self, tokens, parent, q, layer=0, out=None, stream=None):
        """Attention of drafted tokens over the cache, themselves and their ancestors."""
        out = self._check_queries(tokens, q, out, stream)
        self._ints(parent, (tokens.tokens,), "parent")
        self.reserve_tokens_workspace(tokens, self.kv.len + tokens.max_tokens, stream)
        B.dc_tree_attention(self.dims, self.kv, layer, tokens, parent, q, out, self.ws, self.ws_bytes,
                            self._stream_here(stream))
        return out

    def commit_rows(self, tokens, path=None, keep=None, width=None, stream=None):
        """The rows of `tokens`, or of each sequence's `path` [batch][width], join the cache."""
        self._batch_of(tokens)
        if path is not None:
            width = path.shape[1] if path.dim() == 2 else 0
            self._ints(path, (self.dims.batch, width), "path")
        elif width is None:
            width = tokens.max_tokens
        if keep is not None:
            self._ints(keep, (self.dims.batch,), "keep")
        B.dc_commit_rows(self.dims, self.kv, self.feat, tokens, path, keep, width, self._stream_here(stream))

    def tighten_len(self, stream=None) -> int:
        """The bound of the units' rows down to the longest unit's.  commit_rows counts a call's full
        width, as it reads nothing back; where fewer rows stay, the bound would reach the capacity of a
        cache with room, and calls are planned for rows that are not there.  Waits for the stream."""
        if self.unit_len is not None:
            with torch.cuda.stream(stream):            # (None: the current one)
                rows = int(self.unit_len.max())
            self.kv.len = max(0, min(self.kv.len, rows))
        return self.kv.len

    def prefill(self, tokens, rope, q, k, v, pos, layer=0, out=None, stream=None):
        """One layer of a prompt: norm, rotation, the rows into the cache, attention.  After
        the last layer commit_rows(tokens) makes the rows part of the cache."""
        q, _ = self.norm_rope(tokens, rope, q, k, v, pos, layer, stream=stream)
        return self.prompt_attention(tokens, q, layer, out, stream)

    def draft(self, tokens, parent, rope, q, k, v, pos, layer=0, out=None, stream=None):
        """One layer of a tree of drafted tokens: norm, rotation, the rows behind the cache,
        attention.  commit_rows(tokens, path, keep) then keeps the accepted path."""
        q, _ = self.norm_rope(tokens, rope, q, k, v, pos, layer, stream=stream)
        return self.tree_attention(tokens, parent, q, layer, out, stream)

    # ---- rows that sequences share, and blocks of rows

    def reserve_shared_workspace(self, tokens, shared, max_len: int, stream=None):
        """As reserve_tokens_workspace, for shared_attention with prefixes of their present lengths."""
        self._grow(B.dc_shared_workspace_bytes(self.dims, tokens, shared, max_len), stream)

    def shared_attention(self, tokens, shared, q, parent=None, layer=0, out=None, stream=None):
        """prompt_attention (or with `parent` tree_attention) of sequences whose prefixes (make_shared) hold
        rows that they have in common; those are read once for all of them."""
        out = self._check_queries(tokens, q, out, stream)
        if shared.like != self._like_heads() or shared.device != self._device:
            raise ValueError("the prefixes must have the cache's layers, heads, head_dim, dtype and device")
        if shared.sequences > self.dims.batch or (not shared.first and shared.sequences < self.dims.batch):
            raise ValueError(f"prefixes of {shared.sequences} sequences for a cache of {self.dims.batch}")
        if parent is not None:
            self._ints(parent, (tokens.tokens,), "parent")
        shared.update()
        here = self._stream_here(stream)
        self._with_workspace(
            lambda: B.dc_shared_attention(self.dims, self.kv, layer, tokens, parent, shared, q, out, self.ws,
                                          self.ws_bytes, here),
            lambda: self.reserve_shared_workspace(tokens, shared, self.kv.len + tokens.max_tokens, stream))
        return out

    def _with_workspace(self, call, reserve):
        """The call, which enqueues nothing if the workspace is too small; then it grows.  (Asking for the size
        ahead of every call costs the host as much as the call's own plan.)"""
        try:
            call()
        except B.DCError as e:
            if e.status != B.ERR_WORKSPACE:
                raise
            reserve()
            call()

    def _like_heads(self):
        d = self.dims
        return d.n_layers, d.n_q_heads, d.n_kv_heads, d.head_dim, d.dtype

    def make_blocks(self, rows=64) -> B.dc_blocks:
        """Blocks of `rows` rows of this cache, their bounds all zero (block_bounds computes them)."""
        if rows not in (16, 32, 64, 128):
            raise ValueError(f"blocks of {rows} rows: must be 16, 32, 64 or 128")
        x = torch.zeros((self.U, self.cap // rows, 2, self.D), dtype=self.k.dtype, device=self.k.device)
        b = B.dc_blocks(rows, x.data_ptr() or None)
        b.bounds_tensor = x                          # kept alive with b
        return b

    def _blocks_of(self, blocks):
        x = blocks.bounds_tensor
        if x.shape != (self.U, self.cap // blocks.rows, 2, self.D) or x.dtype != self.k.dtype:
            raise ValueError("the blocks are those of another cache")
        self._here(x, "blocks")

    @staticmethod
    def _int32(**numbers):
        """The C structs would take the low 32 bits of larger ones."""
        for name, x in numbers.items():
            if not -2**31 <= x < 2**31:
                raise ValueError(f"{name} = {x} does not fit 32 bits")

    def block_bounds(self, blocks, start=0, stream=None):
        """The bounds of all complete blocks that hold a row from `start` on, every layer's: `start` is the rows
        that the unit with the fewest had at the last call, or 0 after an eviction.  (`len` is those of caches of equal
        lengths; of a ragged cache it is the longest unit's bound, and shorter units' new blocks would be left out.)"""
        self._blocks_of(blocks)
        self._int32(start=start)
        B.dc_block_bounds(self.dims, self.kv, blocks, start, self._stream_here(stream))

    def reserve_block_workspace(self, tokens, blocks, count, max_len: int, share=1, stream=None):
        """As reserve_tokens_workspace, for block_select and block_attention."""
        self._int32(count=count, share=share)
        self._grow(B.dc_block_workspace_bytes(self.dims, tokens, blocks, B.dc_pick(count, share, 0, 0), max_len), stream)

    def _lists(self, tokens, count, share):
        return self.dims.batch, -(-tokens.max_tokens // share), self.dims.n_kv_heads, count

    def block_select(self, tokens, blocks, q, count, share=1, first=0, last=0, layer=0, out=None, stream=None):
        """The `count` blocks that every `share` successive tokens read, for each KV head: the first and last ones
        named so and those whose bound of the queries' logits is the highest.
        Returns int32 [batch][ceil(max_tokens / share)][n_kv_heads][count], ascending, -1 behind."""
        self._batch_of(tokens)
        self._blocks_of(blocks)
        self._like(q, tokens, self.dims.n_q_heads, "q")
        if count < 1 or share < 1:
            raise ValueError("count and share must be at least 1")
        self._int32(count=count, share=share, first=first, last=last)
        shape = self._lists(tokens, count, share)
        if out is not None:
            self._ints(out, shape, "out")
        elif stream is None:
            out = torch.empty(shape, dtype=torch.int32, device=self.k.device)
        else:
            with torch.cuda.stream(stream):
                out = torch.empty(shape, dtype=torch.int32, device=self.k.device)
        here, pick = self._stream_here(stream), B.dc_pick(count, share, first, last)
        self._with_workspace(
            lambda: B.dc_block_select(self.dims, self.kv, layer, tokens, blocks, pick, q, out, self.ws, self.ws_bytes,
                                      here),
            lambda: self.reserve_block_workspace(tokens, blocks, count, self.kv.len + tokens.max_tokens, share, stream))
        return out

    def block_attention(self, tokens, blocks, chosen, q, share=1, layer=0, out=None, stream=None):
        """Causal attention over the chosen blocks (block_select's lists, or another choice in that layout), the
        rows behind the last complete block and the tokens themselves."""
        out = self._check_queries(tokens, q, out, stream)
        self._blocks_of(blocks)
        if share < 1 or chosen.dim() != 4:
            raise ValueError("share must be at least 1 and chosen [batch][groups][n_kv_heads][count]")
        self._int32(share=share)
        count = chosen.shape[3]
        self._ints(chosen, self._lists(tokens, count, share), "chosen")
        here, pick = self._stream_here(stream), B.dc_pick(count, share, 0, 0)
        self._with_workspace(
            lambda: B.dc_block_attention(self.dims, self.kv, layer, tokens, blocks, pick, chosen, q, out, self.ws,
                                         self.ws_bytes, here),
            lambda: self.reserve_block_workspace(tokens, blocks, count, self.kv.len + tokens.max_tokens, share, stream))
        return out

    def sparse_attention(self, tokens, blocks, q, count, share=1, first=0, last=0, layer=0, out=None, stream=None):
        """block_select and block_attention of one layer."""
        chosen = self.block_select(tokens, blocks, q, count, share, first, last, layer, stream=stream)
        return self.block_attention(tokens, blocks, chosen, q, share, layer, out, stream)


def make_shared(prefix: DecodeBuffers, members) -> B.dc_shared:
    """The caches of `prefix` (one sequence each) as rows that sequences of another DecodeBuffers have in common:
    the first members[0] sequences those of prefix 0, the next members[1] those of prefix 1 and so on,
    sequences behind them none.  An int: so many each, which are then all sequences."""
    n = prefix.dims.batch
    equal = isinstance(members, int)
    counts = [members] * n if equal else [int(m) for m in members]
    if len(counts) != n or min(counts) < 0 or max(counts) < 1 or sum(counts) >= 1 << 24:
        raise ValueError(f"members must be the numbers of sequences of {n} prefixes, at least 0, one of them more")
    s = B.dc_shared(ctypes.pointer(prefix.kv), prefix.cap, n, max(counts), None)
    s.prefix = prefix                                # kept alive with s
    s.like, s.device, s.sequences = prefix._like_heads(), prefix._device, sum(counts)
    if not equal:
        first = [0]
        for m in counts:
            first.append(first[-1] + m)
        s.first_tensor = torch.tensor(first, dtype=torch.int32, device=prefix.k.device)
        s.first = s.first_tensor.data_ptr()

    def update():                                    # (shrink moves the rows to other buffers)
        s.capacity = prefix.cap
    s.update = update
    return s


def make_tokens(counts, device="cuda") -> B.dc_tokens:
    """Packed tokens of sequences of `counts` (host) tokens each."""
    counts = [int(c) for c in counts]
    if torch.device(device).type != "cuda":
        raise ValueError(f"the tokens' offsets must be on a GPU, got {device}")
    if not counts or min(counts) < 0 or sum(counts) >= 1 << 31:
        raise ValueError("counts must be one or more numbers of tokens, at least 0, their sum below 2^31")
    most, total = max(counts), sum(counts)
    t = B.dc_tokens(total, most, None)
    t.sequences = len(counts)
    if min(counts) < most:
        cu = [0]
        for c in counts:
            cu.append(cu[-1] + c)
        t.cu_tensor = torch.tensor(cu, dtype=torch.int32, device=device)   # kept alive with t
        t.cu = t.cu_tensor.data_ptr()
        t.device = t.cu_tensor.get_device()
    return t


def make_rope(inv_freq=None, interleaved=False, norm=False, eps=1e-6, q_gain=None, k_gain=None) -> B.dc_rope:
    """Norm and rotation of a head; inv_freq [rot_dim / 2] float32 (None: no rotation), gains
    [head_dim] float32, all on the cache's device."""
    given = [(name, x) for name, x in (("inv_freq", inv_freq), ("q_gain", q_gain), ("k_gain", k_gain))
             if x is not None]
    for name, x in given:
        if x.dtype != torch.float32 or x.dim() != 1 or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 vector")
        if not x.is_cuda or x.device != given[0][1].device:
            raise ValueError(f"{name} is on {x.device}: all must be on the cache's GPU")
    if q_gain is not None and k_gain is not None and q_gain.numel() != k_gain.numel():
        raise ValueError(f"gains of {q_gain.numel()} and {k_gain.numel()} elements")
    r = B.dc_rope(int(norm), eps, B._ptr(q_gain), B._ptr(k_gain),
                  0 if inv_freq is None else 2 * inv_freq.numel(), int(interleaved), B._ptr(inv_freq))
    r.tensors = (inv_freq, q_gain, k_gain)       # kept alive with r
    if given:
        r.device = given[0][1].get_device()
    gain = q_gain if q_gain is not None else k_gain
    if gain is not None:
        r.gain_len = gain.numel()
    return r


def subset_log_prob(scores: torch.Tensor, budget: int, tau: float = 1.0, kept=None, logz=True,
                    stream=None):
    """log Z and (with `kept`) log pi for every row of `scores` ([units][len] float32
    on the device).  Returns (logz, logp) float64 tensors (logp None without kept)."""
    units, length = scores.shape
    dev = scores.device
    lz = torch.empty(units, dtype=torch.float64, device=dev) if logz else None
    lp = torch.empty(units, dtype=torch.float64, device=dev) if kept is not None else None
    need = B.dc_subset_log_prob_workspace_bytes(units, length, budget)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    B.dc_subset_log_prob(units, length, budget, tau, scores, kept, lz, lp, ws, need,
                         stream_handle(stream))
    return lz, lp


def make_policy(params: torch.Tensor, hidden, n_in: int = 4, layer_norm: bool = False) -> B.dc_policy:
    hidden = tuple(hidden)
    h = (ctypes.c_int32 * 2)(hidden[0], hidden[1] if len(hidden) > 1 else 0)
    return B.dc_policy(n_in, len(hidden), h, params.data_ptr(), int(layer_norm))
