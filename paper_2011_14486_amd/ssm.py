"""A state-space value network on the sequence operators.

V(s) is the sum of one prediction per stage, as of the recurrent network.  A stage's features are one token:

    h = W_in x;   per block:  h += W_out norm(scan(W_proj norm(h)));   prediction = w_head norm(h) + b_head

Weights are held in 4 bits, the rows that meet them in 8; the residual stream h is bf16, sums and states are fp32.

`score` takes whole sequences, `extend` one more stage for every row.  Both may begin from states kept per slot and
leave theirs in slots, so that a search scores its prefixes once and then each extension by one token:

    net = SsmValue(ctx, inputs.ssm_weights(64, 256, 2, heads=4))
    prefixes, beam = net.state(64), net.state(1024)
    values = net.score(x, n_seq=64, state_out=prefixes)             # x bf16 [64 T][F]
    values = net.extend(y, prefixes, parents, state_out=beam)       # y bf16 [1024][F], parents int32 [1024]
"""
from __future__ import annotations

from typing import Any, NamedTuple

from . import binding as vf


class SsmState(NamedTuple):
    """Per slot: (conv, ssm) of every block, and the sum of the predictions so far."""
    blocks: Any
    total: Any


def sums_of_ranges(torch, each, offsets):
    """Sums of the sequences' predictions; ranges as the operators take them: one that does not lie in the tokens is empty."""
    tokens = each.shape[0]
    begin, end = offsets[:-1], offsets[1:]
    if tokens == 0 or begin.shape[0] == 0:
        return each.new_zeros(begin.shape[0])
    there = (begin >= 0) & (end >= begin) & (end <= tokens)
    # in the order of their begins, so that begins and ends ascend (segment_reduce looks at nothing); every second segment lies
    # between two ranges
    begin, order = torch.where(there, begin, tokens).sort(stable=True)
    ranges = torch.stack((begin, torch.where(there, end, tokens)[order]), 1).reshape(-1).cummax(0).values
    sums = torch.segment_reduce(each, "sum", offsets=ranges, unsafe=True, initial=0)
    return torch.empty_like(sums[::2]).index_copy_(0, order, sums[::2])


class SsmValue:
    """The network on a context's GPU; `weights` as inputs.ssm_weights makes them."""

    def __init__(self, ctx, weights):
        torch = ctx.torch
        self.ctx, self.torch = ctx, torch
        dev = lambda a: torch.from_numpy(a).to(ctx.device)   # noqa: E731
        four = lambda a: vf.vf_mx_quantize(ctx, dev(a), vf.VF_E2M1)   # noqa: E731
        sizes = [weights[k] for k in ("heads", "head_dim", "groups", "n_state")]
        self.inner = sizes[0] * sizes[1]
        self.w_in, self.gain = four(weights["w_in"]), dev(weights["gain"])
        self.w_head, self.b_head = four(weights["w_head"]), dev(weights["b_head"])
        self.not_there = torch.tensor([float("nan"), float("nan"), 0.0], device=ctx.device)
        self.blocks = []
        for b in weights["blocks"]:
            layer = vf.SsmLayer(*sizes, **{k: dev(b[k]) for k in ("conv_w", "conv_b", "a", "d", "dt_bias")})
            self.blocks.append((dev(b["gain"]), four(b["w_proj"]), layer, dev(b["gain_out"]), four(b["w_out"])))

    def state(self, slots):
        """Zeroed state of `slots` slots: the empty prefix."""
        return SsmState([layer.state(slots, self.torch.bfloat16) for _, _, layer, _, _ in self.blocks],
                        self.torch.zeros(slots, device=self.ctx.device))

    def _tokens(self, x, scan):
        """Predictions [tokens] of x [tokens][F]; scan(block, layer, xbc, dt, z) makes a block's outputs."""
        ctx, inner = self.ctx, self.inner
        h = vf.vf_mx_matmul(ctx, vf.vf_mx_quantize(ctx, x, vf.VF_E4M3), self.w_in)
        out = None
        for k, (gain, w_proj, layer, gain_out, w_out) in enumerate(self.blocks):
            rows, total = vf.vf_rms_norm(ctx, h if out is None else out, gain, residual=None if out is None else h, out_type=vf.VF_E4M3)
            h = h if total is None else total
            proj = vf.vf_mx_matmul(ctx, rows, w_proj)
            y = scan(k, layer, proj[:, inner:inner + layer.channels], proj[:, inner + layer.channels:], proj[:, :inner])
            y, _ = vf.vf_rms_norm(ctx, y, gain_out, out_type=vf.VF_E4M3)
            out = vf.vf_mx_matmul(ctx, y, w_out)
        rows, _ = vf.vf_rms_norm(ctx, h if out is None else out, self.gain, residual=None if out is None else h, out_type=vf.VF_E4M3)
        return vf.vf_mx_matmul(ctx, rows, self.w_head, bias=self.b_head, out_type=vf.VF_FP32)[:, 0]

    def score(self, x, n_seq=1, longest=None, offsets=None, state=None, slots=None, state_out=None, slots_out=None):
        """Values [n_seq] of whole sequences x bf16 [tokens][F]; other arguments as vf_ssm_scan."""
        def scan(k, layer, xbc, dt, z):
            return vf.vf_ssm_scan(self.ctx, layer, xbc, dt, z, n_seq, longest, offsets, None if state is None else state.blocks[k], slots,
                                  None if state_out is None else state_out.blocks[k], slots_out)

        each = self._tokens(x, scan)
        if offsets is None:
            value = each.reshape(n_seq, each.shape[0] // n_seq if n_seq else 0).sum(1)
        else:
            value = self._sums(each, offsets.long())
        return self._totals(value, state, slots, state_out, slots_out)

    def _sums(self, each, offsets):
        return sums_of_ranges(self.torch, each, offsets)

    def extend(self, x, state, slots=None, state_out=None, slots_out=None):
        """Values [rows] with one more stage x bf16 [rows][F]: row r continues slot slots[r] of `state` (-1: the empty prefix) and
        leaves its state in slot slots_out[r] of `state_out` (-1: nowhere)."""
        def scan(k, layer, xbc, dt, z):
            return vf.vf_ssm_step(self.ctx, layer, xbc, dt, z, state.blocks[k], slots, None if state_out is None else state_out.blocks[k], slots_out)

        return self._totals(self._tokens(x, scan), state, slots, state_out, slots_out)

    def _totals(self, value, state, slots, state_out, slots_out):
        """Sums by slots as the operators have them: -1 is the empty prefix, or no place to leave one; a slot that is not there reads as
        NaN and is not written.  (The sums with three numbers behind them: past the end, -2 and -1 as indexes.)"""
        behind = lambda total, k: (self.torch.cat((total, self.not_there)), k.clamp(-2, total.shape[0]).long())   # noqa: E731
        if state is not None:
            if slots is None:
                value = value + state.total[:value.shape[0]]
            else:
                sums, at = behind(state.total, slots)
                value = value + sums[at]
        if state_out is not None:
            if slots_out is None:
                state_out.total[:value.shape[0]] = value
            else:
                sums, at = behind(state_out.total, slots_out)
                sums[at] = value
                state_out.total.copy_(sums[:-3])
        return value
