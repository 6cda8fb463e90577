"""A student without gates that read the state, taught by a GRU: the operators of ops.py as they are used together.

`LinearStudent` is a stack of gated linear recurrent layers with a linear head.  Every layer takes one product
for its gates and candidates, side by side, and runs the recurrence on the two halves:

    (g | v)_t = W x_t + b,   h_t = sigmoid(g_t) h_{t-1} + (1 - sigmoid(g_t)) v_t;

layer j + 1 reads the states of layer j, the head reads the top layer's.

* `teacher_top` makes a teacher's side of the loss from its logits: the top K of every row (`token_logprobs`);
* `step` is a training step: forward (`glr_forward`), loss and gradient with respect to the logits in one pass
  (`distill_topk`), backward (`glr_backward`), torch Adam.  The products of training are torch matrix
  products, as the head of `training.GruStackTrainer` is;
* `Served` is the trained student for serving: its weights in 8 bits (`q8_quantize`), products `q8_linear`; `read`
  takes whole prompts in, `next` one token of each running sequence (`glr_step` on a pool of states), both
  return logits, and `alternatives` scores them (`token_logprobs`).

Teachers are whatever gives logits per position; the states of a GRU layer (`gru_serial_scan`, `mgrit_gru_forward`)
times a head are what this framework trains.  ``python -m paper_2203_04738_amd.student`` runs the whole path on a
small example.
"""
from __future__ import annotations

from . import binding as _b
from . import ops as _o


def _empty(n, like):
    import torch
    return torch.empty(n, dtype=torch.uint8, device=like.device)


def teacher_top(logits, K: int):
    """(ids[N,K], values[N,K]): a teacher's K largest logits of every row, up to a constant of the row (log
    probabilities), as `distill_topk` takes them."""
    import torch
    N, V = logits.shape
    cfg = _o.LogitsCfg(N, V, K, _CODES()[logits.dtype])
    top = torch.empty(N, K, device=logits.device)
    ids = torch.empty(N, K, dtype=torch.int64, device=logits.device)
    _o.token_logprobs(cfg, logits, None, None, None, top, ids, _empty(_o.logits_workspace_bytes(cfg), logits))
    return ids, top


def _CODES():
    import torch
    return {torch.float32: _b.MGRIT_F32, torch.bfloat16: _b.MGRIT_BF16, torch.float16: _o.MGRIT_F16}


class LinearStudent:
    """params: per layer [W[2H,D_j], b[2H]] (gates above candidates), head: [W_o[V,H], b_o[V]]; float32 CUDA
    tensors, updated in place.  T, B: steps and batch of a training step."""

    def __init__(self, T: int, B: int, params, head, *, K: int, temperature: float = 1.0, lr: float = 1e-3):
        import torch
        self.T, self.B = T, B
        self.params, self.head = [list(p) for p in params], list(head)
        self.H, self.V = self.params[0][0].shape[0] // 2, self.head[0].shape[0]
        dev = self.params[0][0].device
        self.cfg = _o.GlrCfg(T, B, self.H)
        self.loss_cfg = _o.LogitsCfg(T * B, self.V, K, _b.MGRIT_F32, temperature)
        z = lambda *s: torch.empty(*s, device=dev)  # noqa: E731
        L, H = len(self.params), self.H
        self.ws = _empty(max(_o.glr_workspace_bytes(self.cfg), _o.logits_workspace_bytes(self.loss_cfg)), z(1))
        self.gv = [z(T, B, 2 * H) for _ in range(L)]           # gates and candidates, and their gradients
        self.dgv = z(T, B, 2 * H)
        self.h = [z(T, B, H) for _ in range(L)]
        self.saved = [_empty(_o.glr_saved_bytes(self.cfg), z(1)) for _ in range(L)]
        self.opt = torch.optim.Adam([q for p in self.params for q in p] + self.head, lr=lr)

    def forward(self, x):
        """States of the top layer [T,B,H] for x[T,B,D]; keeps what `step` differentiates."""
        import torch
        T, B, H = self.T, self.B, self.H
        for j, (W, b) in enumerate(self.params):
            xin = x if j == 0 else self.h[j - 1]
            torch.addmm(b, xin.reshape(T * B, -1), W.t(), out=self.gv[j].view(T * B, 2 * H))
            _o.glr_forward(self.cfg, self.gv[j][..., :H], self.gv[j][..., H:], None, None, self.h[j], None,
                           self.saved[j], self.ws)
        return self.h[-1]

    def logits(self, x):
        h = self.forward(x)
        return h.view(self.T * self.B, self.H) @ self.head[0].t() + self.head[1]

    def step(self, x, ids, values) -> float:
        """One optimiser step on the mean distillation loss against a teacher's (ids, values)[T*B,K] (rows of
        negative ids do not count); returns the loss before the update."""
        import torch
        T, B, H = self.T, self.B, self.H
        n = T * B
        out = self.logits(x)
        rows = (ids >= 0).any(1)
        weight = rows.float() / rows.sum().clamp(min=1)
        loss = torch.empty(n, device=out.device)
        _o.distill_topk(self.loss_cfg, out, ids, values, weight, loss, None, out, self.ws)   # out is its gradient now
        top = self.h[-1].view(n, H)
        self.head[0].grad, self.head[1].grad = out.t() @ top, out.sum(0)
        dh = (out @ self.head[0]).view(T, B, H)
        for j in range(len(self.params) - 1, -1, -1):
            W, b = self.params[j]
            gv, d = self.gv[j], self.dgv
            _o.glr_backward(self.cfg, gv[..., :H], gv[..., H:], None, self.saved[j], dh, None, d[..., :H], d[..., H:],
                            None, self.ws)
            flat = d.view(n, 2 * H)
            xin = (x if j == 0 else self.h[j - 1]).reshape(n, -1)
            W.grad, b.grad = flat.t() @ xin, flat.sum(0)
            if j > 0:
                dh = (flat @ W).view(T, B, H)
        self.opt.step()
        return float((loss * weight).sum())


class Served:
    """A trained student with 8-bit weights and a pool of `slots` running sequences (all start from zero states)."""

    def __init__(self, student: LinearStudent, slots: int):
        import torch
        self.H, self.V = student.H, student.V
        self.layers = [self._pack(W) + (b.clone(),) for W, b in student.params]
        self.head = self._pack(student.head[0]) + (student.head[1].clone(),)
        dev = student.head[0].device
        # (a row more than the pool has, for what `read` leaves of idle rows)
        self._pool = [torch.zeros(slots + 1, self.H, device=dev) for _ in self.layers]
        self.state = [p[:slots] for p in self._pool]

    @staticmethod
    def _pack(W):
        """(q, scale, width) of a weight matrix, a scale per output channel."""
        import torch
        N, K = W.shape
        q = torch.empty(N, _o.q8_row_bytes(K), dtype=torch.int8, device=W.device)
        scale = torch.empty(N, device=W.device)
        _o.q8_quantize(_o.Q8Cfg(N, 1, K), W.contiguous(), q, scale)
        return q, scale, K

    @staticmethod
    def _linear(x, layer):
        import torch
        q, scale, K, bias = layer
        cfg = _o.Q8Cfg(x.shape[0], q.shape[0], K)
        y = torch.empty(x.shape[0], q.shape[0], device=x.device)
        _o.q8_linear(cfg, x, q, scale, bias, y, _empty(_o.q8_workspace_bytes(cfg), x))
        return y

    def read(self, x, slots):
        """Takes prompts x[T,B,D] in from zero states and leaves their states in the pool rows `slots` (int32 [B]; a row
        whose slot is outside the pool is idle, as in `next`: no state is touched); returns the logits [B,V] behind
        their last step."""
        import torch
        T, B, H = x.shape[0], x.shape[1], self.H
        n = len(self.state[0])
        to = torch.where((slots >= 0) & (slots < n), slots, n).long()
        cfg = _o.GlrCfg(T, B, H)
        ws = _empty(_o.glr_workspace_bytes(cfg), x)
        h = x
        for layer, pool in zip(self.layers, self._pool):
            gv = self._linear(h.reshape(T * B, -1), layer).view(T, B, 2 * H)
            h, last = torch.empty(T, B, H, device=x.device), torch.empty(B, H, device=x.device)
            _o.glr_forward(cfg, gv[..., :H], gv[..., H:], None, None, h, last, None, ws)
            pool.index_copy_(0, to, last)
        return self._linear(h[-1], self.head)

    def next(self, x, slots):
        """One step x[B,D] of the sequences in the pool rows `slots`; returns their logits [B,V]."""
        import torch
        H, h = self.H, x
        cfg = _o.GlrCfg(1, x.shape[0], H)
        for layer, state in zip(self.layers, self.state):
            gv = self._linear(h, layer)
            h = torch.empty(x.shape[0], H, device=x.device)
            _o.glr_step(cfg, gv[:, :H], gv[:, H:], slots, None, state, state, h)
        return self._linear(h, self.head)

    def alternatives(self, logits, K: int, tokens=None):
        """(log p of `tokens` or None, entropy, top log p, top ids) of rows of logits."""
        import torch
        N, V = logits.shape
        new = lambda *s, **kw: torch.empty(*s, device=logits.device, **kw)  # noqa: E731
        logp, entropy = None if tokens is None else new(N), new(N)
        top, ids = new(N, K), new(N, K, dtype=torch.int64)
        cfg = _o.LogitsCfg(N, V, K)
        _o.token_logprobs(cfg, logits, tokens, logp, entropy, top, ids, _empty(_o.logits_workspace_bytes(cfg), logits))
        return logp, entropy, top, ids


def example(T: int = 128, B: int = 32, D: int = 12, H: int = 64, V: int = 200, K: int = 8, steps: int = 60, seed: int = 0,
            say=print):
    """A GRU layer with a head as the teacher, a student of two layers taught from its top K logits, served in 8 bits.
    Returns (first loss, last loss, largest difference between the served logits read at once and token by token,
    largest difference to the student's own logits over their spread)."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    gru = [r(3 * H, D) / D ** 0.5, r(3 * H, H) / H ** 0.5, torch.zeros(3 * H, device="cuda"), torch.zeros(3 * H, device="cuda")]
    head = 3 * r(V, H) / H ** 0.5
    cfg = _b.MgritGruCfg(T, B, D, H, propagator=1)
    ws, states = _empty(_b.mgrit_gru_workspace_bytes(cfg), head), torch.empty(T + 1, B, H, device="cuda")

    def batch():
        x = r(T, B, D)
        _b.gru_serial_scan(cfg, *gru, x, torch.zeros(B, H, device="cuda"), states, ws)
        return (x,) + teacher_top(states[1:].reshape(T * B, H) @ head.t(), K)

    params = [[r(2 * H, n) / n ** 0.5, torch.zeros(2 * H, device="cuda")] for n in (D, H)]
    student = LinearStudent(T, B, params, [r(V, H) / H ** 0.5, torch.zeros(V, device="cuda")], K=K, lr=5e-3)
    losses = [student.step(*batch()) for _ in range(steps)]
    say(f"distillation loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps")
    x, _, _ = batch()
    own = student.logits(x).view(T, B, V)[-1]
    served = Served(student, slots=B + 3)
    slots = torch.randperm(B + 3, generator=g, device="cuda")[:B].to(torch.int32)
    at_once = served.read(x, slots)
    for s in served.state:
        s.zero_()
    for t in range(T):
        by_token = served.next(x[t], slots)
    _, entropy, top, ids = served.alternatives(by_token, 3)
    say(f"after {T} tokens: entropy {float(entropy.mean()):.3f}, best token's log probability {float(top[:, 0].mean()):.3f}")
    return (losses[0], losses[-1], float((at_once - by_token).abs().max()),
            float((at_once - own).abs().max() / own.std()))


if __name__ == "__main__":
    print(example())
