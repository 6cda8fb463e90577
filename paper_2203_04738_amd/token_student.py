"""A recurrent student over tokens, taught by imitation and by reward: the operators of token_ops.py as they are used
together, with those of ops.py beside them.

`TokenStudent` reads tokens through an embedding (`embed_lookup`), layers of a short convolution and a selective scan, and
a linear head:

    (x | z) = W_in u,   x' = conv(x),   (dt | b | c) = W_dbc x',   y = scan(x', dt, b, c, z),   u <- u + W_out y.

* `imitate` is a training step on a teacher's top logits (`distill_topk`), `learn` one on rewards (`policy_loss`): both
  give the gradient of the logits in the pass that computes the loss, and go back through `ssm_backward`,
  `causal_conv_backward` and `embed_backward`; the products of training are torch matrix products;
* `act` samples actions and says how probable they were (`token_logprobs`), which is what `learn` compares with later;
* `TokenServed` is the trained student for serving: weights in 8 bits (`q8_linear`), pools of the convolutions' pasts and
  the scans' states; `read` takes whole prompts in, `next` one token of each running sequence (`causal_conv_step`,
  `ssm_step`).

``python -m paper_2203_04738_amd.token_student`` runs the whole path on a small example.
"""
from __future__ import annotations

from . import ops as _o
from . import token_ops as _t
from .student import Served, _empty

NAMES = ("W_in", "conv_w", "conv_b", "W_dbc", "a_log", "dt_bias", "skip", "W_out")


def _new(like, *shape):
    import torch
    return torch.empty(*shape, device=like.device)


def init(V: int, D: int, H: int, S: int, W: int, layers: int, seed: int = 0, device="cuda"):
    """(table, [layer], head) of random weights: decays of 1 to S, steps of 0.001 to 0.1."""
    import math

    import torch
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731

    def layer():
        d = torch.exp(math.log(1e-3) + math.log(100.0) * torch.rand(H, generator=g))
        p = {"W_in": r(2 * H, D) / D ** 0.5, "conv_w": r(H, W) / W ** 0.5, "conv_b": torch.zeros(H),
             "W_dbc": r(H + 2 * S, H) / H ** 0.5, "a_log": torch.log(torch.arange(1, S + 1).float()).repeat(H, 1),
             "dt_bias": d + torch.log(-torch.expm1(-d)), "skip": torch.ones(H), "W_out": r(D, H) / H ** 0.5}
        return {k: v.to(device) for k, v in p.items()}

    return r(V, D).to(device) / D ** 0.5, [layer() for _ in range(layers)], (r(V, D) / D ** 0.5).to(device)


class TokenStudent:
    """table[V,D], layers: a dict of NAMES each, head[V,D]: float32 CUDA tensors, updated in place.  T, B: steps and batch of
    a training step; embeddings are scaled by sqrt(D)."""

    def __init__(self, T: int, B: int, table, layers, head, *, K: int = 1, temperature: float = 1.0,
                 rule: _t.PolicyCfg | None = None, lr: float = 1e-3):
        import torch
        self.T, self.B, self.table, self.layers, self.head = T, B, table, layers, head
        V, D = table.shape
        H, W, S = layers[0]["conv_w"].shape + layers[0]["a_log"].shape[1:]
        self.V, self.D, self.H, self.W, self.S, n = V, D, H, W, S, T * B
        self.embed = _t.EmbedCfg(n, V, D, scale=D ** 0.5)
        self.conv, self.ssm = _t.ConvCfg(T, B, H, W), _t.SsmCfg(T, B, H, S)
        self.rows, self.rule = _o.LogitsCfg(n, V, K, temperature=temperature), rule or _t.PolicyCfg()
        z = lambda *s: _new(head, *s)  # noqa: E731
        self.ws = _empty(max(_t.embed_workspace_bytes(self.embed), _t.causal_conv_workspace_bytes(self.conv),
                             _t.ssm_workspace_bytes(self.ssm), _t.policy_workspace_bytes(self.rows),
                             _o.logits_workspace_bytes(self.rows)), head)
        self.u = [z(T, B, D) for _ in range(len(layers) + 1)]              # before each layer, and behind the last
        self.xz = [z(T, B, 2 * H) for _ in layers]
        self.x = [z(T, B, H) for _ in layers]
        self.dbc = [z(T, B, H + 2 * S) for _ in layers]
        self.y = [z(T, B, H) for _ in layers]
        self.a = [z(H, S) for _ in layers]
        self.saved = [_empty(_t.ssm_saved_bytes(self.ssm), head) for _ in layers]
        self.tokens = self.reset = None
        self.opt = torch.optim.Adam([table, head] + [p[k] for p in layers for k in NAMES], lr=lr)

    def _parts(self, j, xz, x, dbc):
        """What the scan of layer j reads, or what its gradients go to: x, dt, b, c, z."""
        H, S = self.H, self.S
        return x, dbc[..., :H], dbc[..., H:H + S], dbc[..., H + S:], xz[..., H:]

    def logits(self, tokens, reset=None):
        """Logits [T*B,V] behind tokens[T,B] (int64; negative: padding); reset[T,B] bytes: sequences packed one behind the
        other.  Keeps what a training step differentiates."""
        import torch
        T, B, H, n = self.T, self.B, self.H, self.T * self.B
        self.tokens, self.reset = tokens.reshape(n).contiguous(), reset
        _t.embed_lookup(self.embed, self.tokens, self.table, self.u[0].view(n, self.D))
        for j, p in enumerate(self.layers):
            torch.mm(self.u[j].view(n, -1), p["W_in"].t(), out=self.xz[j].view(n, -1))
            _t.causal_conv_forward(self.conv, self.xz[j][..., :H], p["conv_w"], p["conv_b"], None, reset, self.x[j], None)
            torch.mm(self.x[j].view(n, H), p["W_dbc"].t(), out=self.dbc[j].view(n, -1))
            torch.neg(p["a_log"].exp(), out=self.a[j])
            _t.ssm_forward(self.ssm, *self._parts(j, self.xz[j], self.x[j], self.dbc[j]), self.a[j], p["skip"], p["dt_bias"],
                           None, reset, self.y[j], None, self.saved[j], self.ws)
            torch.addmm(self.u[j].view(n, -1), self.y[j].view(n, H), p["W_out"].t(), out=self.u[j + 1].view(n, -1))
        return self.u[-1].view(n, self.D) @ self.head.t()

    def _backward(self, dlogits):
        """Gradients of all weights from those of the logits."""
        T, B, D, H, S, n = self.T, self.B, self.D, self.H, self.S, self.T * self.B
        self.head.grad = dlogits.t() @ self.u[-1].view(n, D)
        du = dlogits @ self.head
        dxz, dx, ddbc = _new(du, T, B, 2 * H), _new(du, T, B, H), _new(du, T, B, H + 2 * S)
        for j in range(len(self.layers) - 1, -1, -1):
            p, a = self.layers[j], self.a[j]
            dy = (du @ p["W_out"]).view(T, B, H)
            g = {k: _new(du, *p[k].shape) for k in ("conv_w", "conv_b", "dt_bias", "skip")}
            da = _new(du, H, S)
            _t.ssm_backward(self.ssm, *self._parts(j, self.xz[j], self.x[j], self.dbc[j]), a, p["skip"], p["dt_bias"], self.reset,
                            self.saved[j], dy, None, *self._parts(j, dxz, dx, ddbc), da, g["skip"], g["dt_bias"], None, self.ws)
            p["W_out"].grad, p["a_log"].grad = du.t() @ self.y[j].view(n, H), da * a
            flat = ddbc.view(n, -1)
            p["W_dbc"].grad = flat.t() @ self.x[j].view(n, H)
            dx.view(n, H).addmm_(flat, p["W_dbc"])
            _t.causal_conv_backward(self.conv, self.xz[j][..., :H], p["conv_w"], p["conv_b"], None, self.reset, dx, None,
                                    dxz[..., :H], g["conv_w"], g["conv_b"], None, self.ws)
            flat = dxz.view(n, 2 * H)
            p["W_in"].grad = flat.t() @ self.u[j].view(n, D)
            du = du + flat @ p["W_in"]
            for k, v in g.items():
                p[k].grad = v
        self.table.grad = _new(du, self.V, D)
        _t.embed_backward(self.embed, self.tokens, du, self.table.grad, self.ws)

    def imitate(self, tokens, ids, values, reset=None) -> float:
        """One optimiser step on the mean distillation loss against a teacher's (ids, values)[T*B,K] (rows of negative ids do
        not count); returns the loss before the update."""
        out = self.logits(tokens, reset)
        rows = (ids >= 0).any(1)
        weight, loss = rows.float() / rows.sum().clamp(min=1), _new(out, len(out))
        _o.distill_topk(self.rows, out, ids, values, weight, loss, None, out, self.ws)     # out is its gradient now
        self._backward(out)
        self.opt.step()
        return float((loss * weight).sum())

    def act(self, tokens, uniform, reset=None):
        """(actions[T*B], their log probabilities): a token sampled behind every step of tokens[T,B] by the numbers
        uniform[T*B] in [0, 1)."""
        import torch
        out = self.logits(tokens, reset)
        p = torch.softmax(out / self.rows.temperature, 1)
        upto = p.cumsum(1)
        # the first token whose sum exceeds the number; a token of no probability, which only sums that rounding leaves out of
        # order could name, gives way to the likeliest
        actions = torch.searchsorted(upto, uniform[:, None] * upto[:, -1:], right=True).clamp(max=self.V - 1)
        actions = torch.where(p.gather(1, actions) > 0, actions, p.argmax(1, keepdim=True))[:, 0]
        return actions, self.log_probs(out, actions)

    def log_probs(self, logits, actions):
        """Log probabilities [T*B] of actions (negative: none, 0) under rows of logits."""
        logp = _new(logits, len(logits))
        cfg = _o.LogitsCfg(len(logits), self.V, 0, temperature=self.rows.temperature)
        _o.token_logprobs(cfg, logits, actions, logp, None, None, None, self.ws)
        return logp

    def learn(self, tokens, actions, old_logp, advantage, ref_logp=None, reset=None):
        """One optimiser step on the mean policy loss of the actions [T*B] (negative: not sampled); returns (loss before the
        update, mean of the KL estimates, share of ratios beyond the clip)."""
        out = self.logits(tokens, reset)
        n = len(out)
        rows = actions >= 0
        weight = rows.float() / rows.sum().clamp(min=1)
        loss, ratio, kl = _new(out, n), _new(out, n), _new(out, n)
        _t.policy_loss(self.rows, self.rule, out, actions, old_logp, ref_logp, advantage, weight, loss, None, ratio, kl, None,
                       out, self.ws)                                                         # out is its gradient now
        self._backward(out)
        self.opt.step()
        beyond = ((ratio < 1 - self.rule.clip_low) | (ratio > 1 + self.rule.clip_high)) & rows
        return float((loss * weight).sum()), float((kl * weight).sum()), float((beyond * weight).sum())


class TokenServed:
    """A trained student with 8-bit weights and pools of `slots` running sequences (all start from nothing)."""

    def __init__(self, student: TokenStudent, slots: int):
        import torch
        s = self.student = student
        self.zero = torch.zeros(max(2 * s.H, s.H + 2 * s.S, s.D, s.V), device=s.head.device)
        pack = lambda w: Served._pack(w) + (self.zero[: w.shape[0]],)  # noqa: E731
        self.layers = [{k: pack(v) if k.startswith("W") else v.clone() for k, v in p.items()} for p in s.layers]
        for p in self.layers:
            p["a"] = -p.pop("a_log").exp()
        self.table, self.head = s.table.clone(), pack(s.head)
        # (a row more than the pools have, for what `read` leaves of idle rows)
        self._past = [torch.zeros(slots + 1, s.W - 1, s.H, device=s.head.device) for _ in self.layers]
        self._state = [torch.zeros(slots + 1, s.H, s.S, device=s.head.device) for _ in self.layers]
        self.past, self.state = [p[:slots] for p in self._past], [p[:slots] for p in self._state]

    def _embed(self, tokens):
        s = self.student
        u = _new(self.table, len(tokens), s.D)
        _t.embed_lookup(_t.EmbedCfg(len(tokens), s.V, s.D, scale=s.D ** 0.5), tokens, self.table, u)
        return u

    def read(self, tokens, slots):
        """Takes prompts tokens[T,B] in from nothing and leaves their pasts and states in the pool rows `slots` (int32 [B]; a
        row whose slot is outside the pool is idle: nothing is touched); returns the logits [B,V] behind the last step."""
        import torch
        T, B = tokens.shape
        H, S, W, n = self.student.H, self.student.S, self.student.W, len(self.state[0])
        to = torch.where((slots >= 0) & (slots < n), slots, n).long()
        conv, ssm = _t.ConvCfg(T, B, H, W), _t.SsmCfg(T, B, H, S)
        ws = _empty(_t.ssm_workspace_bytes(ssm), self.table)
        u = self._embed(tokens.reshape(T * B).contiguous())
        for p, past, state in zip(self.layers, self._past, self._state):
            xz = Served._linear(u, p["W_in"]).view(T, B, 2 * H)
            x, y = _new(u, T, B, H), _new(u, T, B, H)
            last, h_last = _new(u, B, W - 1, H), _new(u, B, H, S)
            _t.causal_conv_forward(conv, xz[..., :H], p["conv_w"], p["conv_b"], None, None, x, last)
            dbc = Served._linear(x.view(T * B, H), p["W_dbc"]).view(T, B, H + 2 * S)
            _t.ssm_forward(ssm, x, dbc[..., :H], dbc[..., H:H + S], dbc[..., H + S:], xz[..., H:], p["a"], p["skip"],
                           p["dt_bias"], None, None, y, h_last, None, ws)
            past.index_copy_(0, to, last)
            state.index_copy_(0, to, h_last)
            u = u + Served._linear(y.view(T * B, H), p["W_out"])
        return Served._linear(u.view(T, B, -1)[-1], self.head)

    def next(self, tokens, slots, reset=None):
        """One token of each of the sequences in the pool rows `slots`; reset[B] bytes: sequences that start anew.  Returns
        their logits [B,V]."""
        B = len(tokens)
        H, S, W = self.student.H, self.student.S, self.student.W
        conv, ssm = _t.ConvCfg(1, B, H, W), _t.SsmCfg(1, B, H, S)
        u = self._embed(tokens)
        for p, past, state in zip(self.layers, self.past, self.state):
            xz = Served._linear(u, p["W_in"])
            x, y = _new(u, B, H), _new(u, B, H)
            _t.causal_conv_step(conv, xz[:, :H], p["conv_w"], p["conv_b"], slots, reset, past, past, x)
            dbc = Served._linear(x, p["W_dbc"])
            _t.ssm_step(ssm, x, dbc[:, :H], dbc[:, H:H + S], dbc[:, H + S:], xz[:, H:], p["a"], p["skip"], p["dt_bias"], slots,
                        reset, state, state, y)
            u = u + Served._linear(y, p["W_out"])
        return Served._linear(u, self.head)


def example(T: int = 64, B: int = 32, V: int = 40, D: int = 32, H: int = 64, S: int = 16, rounds: int = 15, seed: int = 0,
            say=print):
    """A student that is to say the token before the last one: first shown (its teacher's logits name it), then rewarded for
    it.  Returns (mean reward at first, behind the imitation, behind the rewards, largest difference between logits read at
    once and token by token, largest difference to the student's own logits over their spread)."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    student = TokenStudent(T, B, *init(V, D, H, S, 4, 2, seed), K=2, lr=5e-3, rule=_t.PolicyCfg(0.2, 0.28, 0.02))

    def batch():
        tokens = torch.randint(0, V, (T, B), generator=g, device="cuda")
        goal = torch.cat([torch.full((1, B), -1, device="cuda"), tokens[:-1]]).reshape(-1)     # (none at the first step)
        return tokens, goal

    def play():
        tokens, goal = batch()
        actions, logp = student.act(tokens, torch.rand(T * B, generator=g, device="cuda"))
        actions = torch.where(goal >= 0, actions, goal)
        reward = (actions == goal).float()[goal >= 0]
        return tokens, goal, actions, logp, float(reward.mean())

    first = play()[-1]
    for _ in range(rounds):
        tokens, goal = batch()
        ids = torch.stack([goal, torch.where(goal >= 0, torch.randint(0, V, goal.shape, generator=g, device="cuda"), -1)], 1)
        student.imitate(tokens, ids, torch.tensor([[2.0, 0.0]], device="cuda").expand(T * B, 2).contiguous())
    shown = play()[-1]
    ref = TokenStudent(T, B, student.table.clone(), [{k: v.clone() for k, v in p.items()} for p in student.layers],
                       student.head.clone())
    for _ in range(rounds):
        tokens, goal, actions, logp, reward = play()
        advantage = (actions == goal).float() - reward
        ref_logp = ref.log_probs(ref.logits(tokens), actions)
        for _ in range(2):
            loss, kl, beyond = student.learn(tokens, actions, logp, advantage, ref_logp)
    last = play()[-1]
    say(f"mean reward {first:.3f}, shown {shown:.3f}, rewarded {last:.3f}; KL {kl:.4f}, clipped {beyond:.3f}")
    served = TokenServed(student, slots=B + 3)
    slots = torch.randperm(B + 3, generator=g, device="cuda")[:B].to(torch.int32)
    tokens, _ = batch()
    own = student.logits(tokens).view(T, B, V)[-1]
    at_once = served.read(tokens, slots)
    start = torch.ones(B, dtype=torch.uint8, device="cuda")
    for t in range(T):
        by_token = served.next(tokens[t].contiguous(), slots, start if t == 0 else None)
    return (first, shown, last, float((at_once - by_token).abs().max()),
            float((at_once - own).abs().max() / own.std()))


if __name__ == "__main__":
    print(example())
