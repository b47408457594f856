"""One policy-gradient step through a replayed MoE layer, with the training-side operators.

A tiny policy (token embedding, one MoE layer with a residual, output head) is rolled out once: the
predicted route and the sampled tokens' log-probabilities are recorded.  Then a few inner updates
replay the recorded route, as Algorithm 3 of arxiv 2606.00395 does, with a clipped loss and a KL term:

    forward   pr2_route_replay -> pr2_token_sort -> expert products, pr2_swiglu_checkpoint
              -> pr2_token_unsort -> head -> pr2_policy_loss (which leaves the logits' gradient)
    backward  pr2_token_unsort_backward -> pr2_swiglu_checkpoint_backward, expert products
              -> pr2_token_sort_backward, pr2_replay_gates_backward -> router

Between forward and backward the experts' inputs to the activation are kept in 8 bits only, and the
sorted rows not at all: they are sorted again from the tokens by the same plan.  The experts' matrix
products and their gradients are plain matrix products per expert.

    python examples/replay_training_step.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_00395_gb300 import binding as B  # noqa: E402

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


class ReplayedLayer:
    """Forward and backward pass of the MoE layer on a recorded route (Eq. pr2_output)."""

    def __init__(self, T, d, N, k, m, dtype):
        self.T, self.d, self.N, self.k, self.m, self.dt = T, d, N, k, m, DT[dtype]
        self.dims = B.dims(T, d, N, k, m, 0, dtype)
        self.act_dims = B.act_dims(T * k, m, dtype, ld=2 * m)
        F = T * k
        self.gates, self.probs = self._new(T, k, dt=torch.float32), self._new(T, N, dt=torch.float32)
        self.offsets, self.perm, self.inv = (self._new(n, dt=torch.int32) for n in (N + 1, F, F))
        self.q = self._new(F, 2, m, dt=torch.int8)
        self.scale = self._new(F, 2, -(-m // B.PR2_CKPT_GROUP), dt=torch.float32)
        self.plan_ws = B.alloc_token_workspace(self.dims)

    def _new(self, *shape, dt=None):
        return torch.empty(*shape, dtype=dt or self.dt, device="cuda")

    def _experts(self):
        """(expert, rows) of the sorted batch."""
        at = self.offsets.tolist()
        return [(e, slice(at[e], at[e + 1])) for e in range(self.N) if at[e + 1] > at[e]]

    def forward(self, h, idx, W):
        F, m = self.T * self.k, self.m
        B.check(B.pr2_route_replay(self.dims, h, W["router"], idx, self.gates, self.probs), "pr2_route_replay")
        x = self._new(F, self.d)
        B.check(B.pr2_token_sort(self.dims, h, idx, x, self.offsets, self.perm, self.inv, self.plan_ws),
                "pr2_token_sort")
        both, act, self.y = self._new(F, 2 * m), self._new(F, m), self._new(F, self.d)
        for e, rows in self._experts():
            torch.mm(x[rows], W["gate"][e].t(), out=both[rows, :m])
            torch.mm(x[rows], W["up"][e].t(), out=both[rows, m:])
        B.check(B.pr2_swiglu_checkpoint(self.act_dims, both[:, :m], both[:, m:], act, self.q, self.scale),
                "pr2_swiglu_checkpoint")
        for e, rows in self._experts():
            torch.mm(act[rows], W["down"][e].t(), out=self.y[rows])
        out = torch.empty_like(h)
        B.check(B.pr2_token_unsort(self.dims, self.y, self.gates, self.inv, out), "pr2_token_unsort")
        return out

    def backward(self, h, idx, W, dout):
        """Gradients of the weights (a dict like W) and of h."""
        F, m = self.T * self.k, self.m
        dy, dgates = self._new(F, self.d), torch.empty_like(self.gates)
        B.check(B.pr2_token_unsort_backward(self.dims, dout, self.y, self.gates, self.inv, self.offsets, dy,
                                            dgates), "pr2_token_unsort_backward")
        x, dact, dboth = self._new(F, self.d), self._new(F, m), self._new(F, 2 * m)
        B.check(B.pr2_token_sort(self.dims, h, None, x, self.offsets, None, self.inv), "pr2_token_sort")
        for e, rows in self._experts():
            torch.mm(dy[rows], W["down"][e], out=dact[rows])
        act = self._new(F, m)
        B.check(B.pr2_swiglu_checkpoint_backward(self.act_dims, dact, self.q, self.scale, dboth[:, :m],
                                                 dboth[:, m:], act), "pr2_swiglu_checkpoint_backward")
        grads = {n: torch.zeros(W[n].shape, device="cuda") for n in ("gate", "up", "down")}
        dx = self._new(F, self.d)
        for e, rows in self._experts():
            dg, du = dboth[rows, :m], dboth[rows, m:]
            dx[rows] = dg @ W["gate"][e] + du @ W["up"][e]
            grads["gate"][e], grads["up"][e] = dg.t() @ x[rows], du.t() @ x[rows]
            grads["down"][e] = dy[rows].t() @ act[rows]
        dh = torch.empty_like(h)
        B.check(B.pr2_token_sort_backward(self.dims, dx, self.inv, dh), "pr2_token_sort_backward")
        dlogits = torch.empty_like(self.probs)
        B.check(B.pr2_replay_gates_backward(self.dims, self.probs, idx, dgates, dlogits),
                "pr2_replay_gates_backward")
        grads["router"] = dlogits.t() @ h.float()
        return grads, dh.float() + dlogits @ W["router"].float()


def init(T, d, N, k, m, V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    W = {"router": (N, d), "pred": (N, d), "gate": (N, m, d), "up": (N, m, d), "down": (N, d, m), "embed": (V, d),
         "head": (V, d)}
    std = {"router": 0.1, "pred": 0.01, "embed": 1.0, "head": 0.1}
    W = {n: (std.get(n, 0.05) * torch.randn(*s, generator=g)).to(DT[dtype]).cuda() for n, s in W.items()}
    tokens = torch.randint(0, V, (T,), generator=g).cuda()
    return W, tokens, g


def loss_and_grads(layer, W, tokens, idx, rollout, kl_coef=0.02):
    """Loss [4] and the gradients of every weight on the recorded route."""
    T, V = tokens.numel(), W["head"].shape[0]
    h = W["embed"][tokens]
    out = layer.forward(h, idx, W)
    z = h + out
    logits = z @ W["head"].t()
    dm = B.policy_dims(T, V, "bf16" if h.dtype == torch.bfloat16 else "fp32", clip_low=0.2, clip_high=0.28,
                       kl_coef=kl_coef)
    loss, logp = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    B.check(B.pr2_policy_loss(dm, logits, rollout["actions"], rollout["weight"], rollout["advantage"],
                              rollout["logp"], rollout["logp"], loss, logp, None, logits,
                              B.alloc_policy_workspace(dm)), "pr2_policy_loss")
    dz = logits @ W["head"]  # the loss left its gradient in place of the logits
    grads, dh = layer.backward(h, idx, W, dz)
    grads["head"] = logits.t().float() @ z.float()
    grads["embed"] = torch.zeros(W["embed"].shape, device="cuda").index_add_(0, tokens, dz.float() + dh)
    return loss, grads, out


def roll_out(W, tokens, dims, g):
    """The route predicted and recorded, actions sampled, their log-probabilities."""
    T, V = tokens.numel(), W["head"].shape[0]
    h = W["embed"][tokens]
    idx, gates, _ = B.alloc_route(dims)
    out = torch.empty_like(h)
    B.check(B.pr2_moe_rollout_forward(dims, h, W["router"], W["pred"], idx, gates, None, None, W["gate"], W["up"],
                                      W["down"], None, None, None, out, workspace=B.alloc_workspace(dims)),
            "pr2_moe_rollout_forward")
    probs = torch.softmax(((h + out) @ W["head"].t()).float(), 1)
    actions = torch.multinomial(probs.cpu(), 1, generator=g)[:, 0].cuda()
    logp = probs.gather(1, actions[:, None])[:, 0].log()
    advantage = torch.where(actions < V // 2, 1.0, -1.0)  # the reward: tokens of the lower half
    return idx, dict(actions=actions.int(), logp=logp, advantage=advantage - advantage.mean(), weight=None)


def main(steps=8, T=512, d=256, N=16, k=4, m=192, V=1000, dtype="bf16", seed=0, lr=0.1, log=print):
    W, tokens, g = init(T, d, N, k, m, V, dtype, seed)
    layer = ReplayedLayer(T, d, N, k, m, dtype)
    idx, rollout = roll_out(W, tokens, layer.dims, g)
    losses = []
    for step in range(steps):
        loss, grads, _ = loss_and_grads(layer, W, tokens, idx, rollout)
        for n, grad in grads.items():
            W[n] = (W[n].float() - lr * grad).to(W[n].dtype)
        losses.append(loss.tolist())
        log("update %d: loss %+.4f  policy %+.4f  KL %.4f  clipped %.3f" % (step, *losses[-1]))
    return losses


if __name__ == "__main__":
    main()
