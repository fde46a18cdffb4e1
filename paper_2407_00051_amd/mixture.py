"""A mixture of generators: a router gives every noise row to `top` of the stack's members,
and the row's parameters are the weighted mean of theirs.  Where an inverse problem
has several solutions a single generator settles on one or averages them; members
can each take one.

Forward, on noise n [k][in]:
  1. logits = n Wr^T + br, [k][M]
  2. the row's `top` most likely members and their log probabilities   sagips_choice_logprob
  3. weights: those probabilities, among themselves                     sagips_choice_logprob
  4. rows sorted by member                                              sagips_route, sagips_dispatch
  5. every member on its own rows: 1 + softplus(G_m(n))                 sagips_gen_forward_routed
  6. theta = the weighted sum, rows back in order                       sagips_combine
Backward, from dL/dtheta [k][out]: the same calls' gradients in turn, and with
`entropy_coef` the gradient of -entropy_coef * (mean entropy of the router), which
keeps it from settling before its members differ.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Sequence

from . import Context


class Mixture:
    """Members W, b (stacks [M][..], as Context.gen_forward takes them), router Wr [M][in] and br [M]; all
    updated by the caller.  The gradients of the last backward call are dW, db, dWr, dbr."""

    def __init__(self, ctx: Context, W: Sequence, b: Sequence, Wr, br, top: int = 2, slope: float = 0.2,
                 entropy_coef: float = 0.0):
        import torch
        self.ctx, self.W, self.b, self.Wr, self.br = ctx, list(W), list(b), Wr, br
        self.M = Wr.shape[0]
        if self.W[0].dim() != 3 or self.W[0].shape[0] != self.M or br.shape[0] != self.M:
            raise ValueError("members and router must have the same number of members")
        if not 1 <= top <= min(self.M, 32):
            raise ValueError(f"top must be in [1, {min(self.M, 32)}]")
        self.top, self.slope, self.entropy_coef = int(top), slope, entropy_coef
        self.dW, self.db = [torch.empty_like(w) for w in self.W], [torch.empty_like(v) for v in self.b]
        self.dWr, self.dbr = torch.empty_like(Wr), torch.empty_like(br)
        self._held, self._marked = None, None

    def parameters(self):
        return [t for pair in zip(self.W, self.b) for t in pair] + [self.Wr, self.br]

    def gradients(self):
        return [t for pair in zip(self.dW, self.db) for t in pair] + [self.dWr, self.dbr]

    def on_stream(self):
        """The context's stream as torch's current one: what torch computes here stands between the library's calls."""
        import torch
        return nullcontext() if self.ctx._follow else torch.cuda.stream(self.ctx.stream)

    def _take(self, *inputs):
        """Marks what the context's stream uses and torch's current one may own: inputs, and once a stream the parameters
        and gradients (a mark lasts as long as the memory)."""
        import torch
        c = self.ctx
        if c._follow or torch.cuda.current_stream(c.device).cuda_stream == c.stream.cuda_stream:
            return
        c._owned(*inputs)
        if self._marked is not c.stream:
            c._owned(self.parameters(), self.gradients())
            self._marked = c.stream

    def hand_out(self, *results):
        """Marks what was allocated under on_stream() as used by the caller's stream: the caller may drop it at any time.
        Called outside on_stream(), where that stream is torch's current one."""
        import torch
        if not self.ctx._follow:
            for t in results:
                if t is not None:
                    t.record_stream(torch.cuda.current_stream(self.ctx.device))

    def forward(self, noise):
        """theta [k][out]; what backward needs is kept until the next call.  A row whose logits hold a NaN or +inf
        has no members: its theta is NaN, not the 0 of an empty sum."""
        import torch
        c = self.ctx
        self._take(noise)
        with self.on_stream():
            logits = torch.addmm(self.br, noise, self.Wr.t())
            chosen = c.choice_logprob(logits, top=self.top)
            own = c.choice_logprob(chosen["top_logp"], top=self.top)   # already in falling order: choice i is the i-th
            weight = own["top_logp"].exp()
            plan = c.route(chosen["top_choice"], self.M)
            x = c.dispatch(noise, plan)
            theta = c.gen_forward_routed(self.W, self.b, x, plan["offsets"], slope=self.slope)
            self._held = (noise, logits, chosen, own, weight, plan, x, theta)
            nan = chosen["entropy"][:, None]                           # finite otherwise
            out = c.combine(theta, plan, weight).addcmul_(nan, nan, value=0.0)
        self.hand_out(out)
        return out

    def backward(self, dL_dtheta) -> None:
        """The gradients of the last forward call's parameters from dL/dtheta [k][out]."""
        import torch
        c = self.ctx
        noise, logits, chosen, own, weight, plan, x, theta = self._held
        self._take(dL_dtheta)
        with self.on_stream():
            d_member, d_weight = c.combine_backward(dL_dtheta, theta, plan, weight)
            c.gen_backward_routed(self.W, self.b, x, plan["offsets"], d_member, slope=self.slope, dW=self.dW, db=self.db)
            d_top = c.choice_backward(chosen["top_logp"], own, d_top=d_weight * weight)
            d_entropy = torch.full_like(chosen["entropy"], -self.entropy_coef / noise.shape[0]) if self.entropy_coef else None
            d_logits = c.choice_backward(logits, chosen, d_top=d_top, d_entropy=d_entropy)
            # (one product for both: a library's sum over many rows may clear memory first, which graphs replay wrongly)
            d = torch.mm(d_logits.t(), torch.cat([noise, torch.ones_like(noise[:, :1])], 1))
            self.dWr.copy_(d[:, :-1])
            self.dbr.copy_(d[:, -1])
