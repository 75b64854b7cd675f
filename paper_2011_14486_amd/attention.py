"""An attention value network on the attention operators.

V(s) is the sum of one prediction per stage, as of the recurrent networks.  A stage's features are one token:

    h = W_in x;   per block:  h += W_out attend(W_qkv norm(h)),  h += W_down relu(W_up norm(h));   prediction = w_head norm(h) + b_head

A stage attends to itself and the stages before it, by their positions.  Weights are held in 4 bits, the rows that meet them in 8; the
residual stream h, queries, keys and values are bf16 (keys and values in 8 bits if asked for), sums are fp32.

`score` takes whole sequences, `extend` one more stage for every row, `fork` makes rows that go on from others: they share
the full pages of what they have in common, so that a search scores its prefixes once and then each extension by one token:

    net = AttentionValue(ctx, inputs.attention_weights(64, 256, 2, heads=4, hidden=512))
    state = net.state(1024, stages=100)
    values = net.score(x, n_seq=64, state=state)      # x bf16 [64 T][F]: 64 prefixes
    net.fork(state, parents)                          # parents int32 [1024]: 1024 rows behind them
    values = net.extend(y, state)                     # y bf16 [1024][F]
    net.fork(state, best)                             # best int32 [64]: the rows that the search goes on with
"""
from __future__ import annotations

from . import binding as vf
from .ssm import sums_of_ranges


class AttentionState:
    """What the rows of a search have behind them: a cache per block, the rows' pages, their lengths and the sums of their predictions.

    rows: at most this many at a time; stages: no row gets longer.  `longest` is the longest length that a row may have, as far as the host knows:
    it grows with the calls, and is looked up on the GPU where it would leave no place.  Once a graph holds a call (`captured`) its replays
    add what the host does not know of: then a row without a place has NaN as its value from there on, and is not lengthened."""

    def __init__(self, torch, caches, rows, wide, device):
        self.caches, self.page, self.rows, self.wide, self.longest = caches, caches[0].page, rows, wide, 0
        self.table = torch.arange(rows * wide, dtype=torch.int32, device=device).reshape(rows, wide)
        self.lengths = torch.zeros(rows, dtype=torch.int32, device=device)
        self.total = torch.zeros(rows, device=device)
        self.captured = False


class AttentionValue:
    """The network on a context's GPU; `weights` as inputs.attention_weights makes them."""

    def __init__(self, ctx, weights, interleaved=False, magnitude=1.0):
        torch = ctx.torch
        self.ctx, self.torch = ctx, torch
        dev = lambda a: torch.from_numpy(a).to(ctx.device)   # noqa: E731
        four = lambda a: vf.vf_mx_quantize(ctx, dev(a), vf.VF_E2M1)   # noqa: E731
        self.heads, self.kv_heads, self.head_dim = (weights[k] for k in ("heads", "kv_heads", "head_dim"))
        self.rope = vf.Rope(dev(weights["freq"]), interleaved, magnitude)
        self.w_in, self.gain = four(weights["w_in"]), dev(weights["gain"])
        self.w_head, self.b_head = four(weights["w_head"]), dev(weights["b_head"])
        self.not_there = torch.zeros(3, dtype=torch.int32, device=ctx.device), torch.tensor([float("nan"), float("nan"), 0.0], device=ctx.device)
        self.blocks = [(dev(b["gain"]), four(b["w_qkv"]), four(b["w_out"]),
                        (dev(b["gain_up"]), four(b["w_up"]), four(b["w_down"])) if weights["hidden"] else None) for b in weights["blocks"]]

    def state(self, rows, stages, page=16, fmt=vf.VF_BF16):
        """State of `rows` rows that have nothing behind them; pages of `page` stages, keys and values in fmt (VF_BF16 or VF_E4M3)."""
        if rows < 1 or stages < 1:
            raise ValueError("a row and a stage at least are wanted")
        wide = -(-stages // page)
        caches = [vf.KvCache.zeros(fmt, rows * wide, page, self.kv_heads, self.head_dim, self.ctx.device) for _ in self.blocks or [None]]
        return AttentionState(self.torch, caches, rows, wide, self.ctx.device)

    def _capturing(self):
        """Whether torch's current stream is being captured, so that nothing can be looked up."""
        return self.torch.cuda.is_current_stream_capturing()

    def _tokens(self, x, caches, table, lengths, offsets, longest, longest_kv):
        """Predictions [tokens] of x [tokens][F], the last tokens of sequences of these lengths."""
        ctx, head = self.ctx, self.head_dim
        inner, each = self.heads * head, self.kv_heads * head
        h, out = vf.vf_mx_matmul(ctx, vf.vf_mx_quantize(ctx, x, vf.VF_E4M3), self.w_in), None

        def normed(gain):
            nonlocal h
            rows, total = vf.vf_rms_norm(ctx, h if out is None else out, gain, residual=None if out is None else h, out_type=vf.VF_E4M3)
            h = h if total is None else total
            return rows

        for (gain, w_qkv, w_out, up), cache in zip(self.blocks, caches):
            qkv = vf.vf_mx_matmul(ctx, normed(gain), w_qkv)
            q = qkv[:, :inner]
            vf.vf_kv_append(ctx, cache, qkv[:, inner:inner + each], qkv[:, inner + each:], table, lengths, q=q, rope=self.rope, offsets=offsets,
                            longest=longest, q_out=q)
            y = vf.vf_kv_attend(ctx, cache, q, table, lengths, offsets=offsets, longest=longest, longest_kv=longest_kv)
            out = vf.vf_mx_matmul(ctx, vf.vf_mx_quantize(ctx, y, vf.VF_E4M3), w_out)
            if up is not None:
                gain_up, w_up, w_down = up
                u = vf.vf_mx_matmul(ctx, normed(gain_up), w_up)
                out = vf.vf_mx_matmul(ctx, vf.vf_mx_quantize(ctx, u.relu_(), vf.VF_E4M3), w_down)
        return vf.vf_mx_matmul(ctx, normed(self.gain), self.w_head, bias=self.b_head, out_type=vf.VF_FP32)[:, 0]

    def score(self, x, n_seq=1, longest=None, offsets=None, state=None):
        """Values [n_seq] of whole sequences x bf16 [tokens][F]: sequence s has rows offsets[s] .. offsets[s + 1] - 1 (int32 [n_seq + 1]; None:
        all have tokens / n_seq), behind row s of `state`, which then has them too.  longest: with offsets, no sequence has more tokens, and one that has
        is not taken: its value is NaN (default: looked up on the GPU, in a captured call all tokens).  Without a state every sequence begins from nothing
        and nothing is kept."""
        torch, tokens = self.torch, x.shape[0]
        if n_seq == 0 or tokens == 0:
            return x.new_zeros(n_seq, dtype=torch.float32) if state is None else state.total.clone()
        over = None   # sequences that are not taken
        if offsets is None:
            if tokens % n_seq:
                raise ValueError(f"{tokens} rows cannot be dealt to {n_seq} sequences; offsets are wanted")
            counts = torch.full((n_seq,), tokens // n_seq, dtype=torch.int32, device=self.ctx.device)
            longest = tokens // n_seq
        else:
            begin, end = offsets[:-1], offsets[1:]
            counts = torch.where((begin >= 0) & (end >= begin) & (end <= tokens), end - begin, 0).to(torch.int32)
            if longest is not None:
                over = counts > longest
            elif not self._capturing():
                longest = int(counts.max())
            longest = tokens if longest is None else min(longest, tokens)
        if state is None:
            # (one cache does for all blocks: a block's keys are not looked at after it)
            wide = max(1, -(-longest // 16))
            pages, least = n_seq * wide, tokens // 16 + n_seq
            if pages <= 2 * least:
                table = torch.arange(pages, dtype=torch.int32, device=self.ctx.device).reshape(n_seq, wide)
            else:
                # most sequences are much shorter than the longest: each has as many pages as it needs, at most one more than its tokens fill, the
                # last of them first
                ends = ((counts + 15) >> 4).cumsum(0, dtype=torch.int32)
                pages, table = least, ends[:, None] + torch.arange(-1, -1 - wide, -1, dtype=torch.int32, device=self.ctx.device)
            new = [self.ctx.empty((pages, self.kv_heads, 16, (self.head_dim + 7) // 8 * 8), torch.bfloat16) for _ in range(2)]
            caches = [vf.KvCache(vf.VF_BF16, self.head_dim, *new)] * len(self.blocks)
            lengths, longest_kv = counts, longest
        else:
            if state.lengths.shape[0] != n_seq:
                raise ValueError(f"the state has {state.lengths.shape[0]} rows, not {n_seq}")
            longest_kv, room = state.longest + longest, state.wide * state.page
            caches, table, lengths = state.caches, state.table, state.lengths + counts
            state.captured = state.captured or self._capturing()
            if state.captured:
                over = lengths > room if over is None else over | (lengths > room)
                longest_kv = min(longest_kv, room)
            elif longest_kv > room:
                longest_kv = int(lengths.max())   # (rows have forked to shorter ones, or others have been the longest in turn)
                if longest_kv > room:
                    raise ValueError(f"the state has place for {room} stages a row, not {longest_kv}")
        # (a row of length 0 has no positions: its tokens are written nowhere and see nothing.  Without a state pages are a sequence's own)
        where = lengths if over is None or state is None else torch.where(over, 0, lengths)
        each = self._tokens(x, caches, table, where, offsets, longest, longest_kv)
        value = each.reshape(n_seq, -1).sum(1) if offsets is None else sums_of_ranges(torch, each, offsets.long())
        if over is not None:
            value.masked_fill_(over, float("nan"))
        if state is not None:
            value = value + state.total
            state.total.copy_(value)
            state.lengths.copy_(lengths if over is None else torch.where(over, state.lengths, lengths))
            state.longest = longest_kv
        return value

    def extend(self, x, state):
        """Values [rows] with one more stage x bf16 [rows][F] of every row of `state`, which then has it too."""
        return self.score(x, state.lengths.shape[0], state=state)

    def fork(self, state, parents):
        """Row r of the state goes on from what row parents[r] (int32 or int64 [n], n at most state.rows) has had, as many rows as there are
        parents; -1: from nothing; any other parent that is no row makes a row whose values are NaN.  Full pages are shared, the page that a row goes on in is its own.  The state has other tables and lengths afterwards, and pages that
        no row has are written over, so that a graph holds extensions, not forks."""
        torch, wide, page = self.torch, state.wide, state.page
        n, device = parents.shape[0], self.ctx.device
        if n > state.rows:
            raise ValueError(f"the state has place for {state.rows} rows, not {n}")
        # (lengths and sums with three numbers behind them: past the end, -2 and -1 as indexes)
        rows = state.lengths.shape[0]
        at = parents.clamp(-2, rows).long()
        lengths, total = (torch.cat((have, ends))[at] for have, ends in zip((state.lengths, state.total), self.not_there))
        old = state.table[at.clamp(0, rows - 1)] if rows else state.table.new_zeros((n, wide))
        full = (lengths // page).long()
        at = torch.arange(wide, device=device)
        own = at >= full[:, None]
        # pages that no row shares, in the order of their numbers: there are rows * wide pages, so that there are enough
        used = torch.zeros(state.rows * wide + 1, dtype=torch.int8, device=device)
        used.scatter_(0, torch.where(own, state.rows * wide, old.long()).reshape(-1), 1)
        free = used[:-1].argsort(stable=True)
        turn = (own.reshape(-1).cumsum(0) - 1).clamp(min=0).reshape(n, wide)
        table = torch.where(own, free[turn].to(torch.int32), old)
        # the page that is full in part is copied; where none is, a page to itself
        tail = full.clamp(max=wide - 1)[:, None]
        to = table.gather(1, tail)[:, 0].long()
        source = torch.where((lengths % page != 0) & (full < wide), old.gather(1, tail)[:, 0].long(), to)
        for cache in state.caches:
            for pool in cache.tensors:
                if pool is not None:
                    pool.index_copy_(0, to, pool.index_select(0, source))
        state.table, state.lengths, state.total = table, lengths, total
