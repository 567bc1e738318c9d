"""One DP-SGD-RC training step (Alg. DP-SGD-RC) around libdprc.

Per step:

1. forward with hooks: each trained bias-free linear layer keeps its input A
   ([B, T, d]) and its output S ([B, T, p]);
2. one autograd pass from the summed per-sample losses to the layer outputs
   gives E = dL/dS for every layer (the backward-hook step of the algorithm;
   sample i's rows of E are dL_i/dS_i because samples do not interact, and
   no weight gradient is formed);
3. ``dprc_norm_hutch`` (or ``dprc_norm_hutchpp``) estimates every sample's
   squared gradient norm summed over the layers; adjacent layers that read
   the same activations (q, k, v; gate, up) share one pass over A;
4. ``dprc_clip_scale``: c_i = min(1, C / sqrt(n_i));
5. ``dprc_clip_accumulate_layers``: each layer's clipped gradient sum_i c_i A_i^T E_i
   is formed directly on the matrix cores.  For a linear layer it equals the
   weight gradient of the scaled loss sum_i c_i L_i, i.e. the algorithm's
   second backward pass, without running it;
6. ``dprc_add_noise``: + sigma C N(0, I) per element of the summed gradient;
7. AdamW on fp32 master weights (kept in the [d, p] layout of the clipped
   gradient) with the private gradient divided by the batch size, then the
   bf16 weights are refreshed from the masters.  By default steps 6 and 7
   run as one ``dprc_private_adamw`` pass per layer (noise, division, AdamW
   and the transposed bf16 weight write); ``fused_adamw=False`` runs
   ``dprc_add_noise`` and ``torch.optim.AdamW`` instead.

Only the listed linear layers are trained, and the norms given as ``norms``;
every other parameter (embedding, other norms) is held fixed.  Probes, noise
and the masks of every ``junction`` module that the loss runs are keyed by a
per-step seed derived from (seed, step), so they are fresh every step.

With ``norms`` (``junction.Junction`` modules), step 2 goes on through the first
norm; the backward calls write every sample's weight and bias gradients side by
side into one [B, N] matrix, which goes with the layers' pairs; step 3 starts from its rows' exact squared norms
(``dprc_norm_vectors``), step 5 adds its clipped sum
(``dprc_clip_accumulate_vectors``), and steps 6 and 7 treat all of them as one
more layer, without weight decay.
"""

import torch

from . import dprc as D
from . import junction

_GOLDEN = 0x9E3779B97F4A7C15


def _rows(x):
    B, T, n = x.shape
    return x if x.stride(2) == 1 and x.stride(0) == T * x.stride(1) else x.contiguous()


def step_seed(seed, step):
    """The key of step ``step``: seed + step * 0x9E3779B97F4A7C15 mod 2^64."""
    return (int(seed) + int(step) * _GOLDEN) & 0xFFFFFFFFFFFFFFFF


class Pairs(list):
    """What a capture gives: (A, E, layer) of every trained layer, and in ``vectors`` the per-sample
    gradients [B, N] of the trained norms (None where there are none).  Whoever makes another list of
    them for a step with norms hands ``vectors`` on."""

    def __init__(self, items=(), vectors=None):
        super().__init__(items)
        self.vectors = vectors


class DPSGDRC:
    """DP-SGD with randomized clipping for a model's bias-free linear layers.

    ``linears``: the trained ``nn.Linear`` modules (bias-free), in model order
    so that layers reading the same input are adjacent.  ``estimator``:
    "hutch" (k probes, ``probe`` "rademacher" or "gaussian") or "hutchpp"
    (sketch s, residual probes r).  ``C``: clipping threshold; ``sigma``:
    noise multiplier.  AdamW hyper-parameters as in ``torch.optim.AdamW``.
    ``norms``: the ``junction.Junction`` modules whose weights and biases are
    trained too (parameters of one dtype; they become views of one buffer).
    ``junction`` modules that run in a step take its key for their masks; those in
    ``dropouts`` (and ``norms``) do so also where a caller has set their ``seed``.
    """

    def __init__(self, linears, C, sigma, estimator="hutch", k=16, probe="rademacher", s=16, r=32,
                 side=D.SIDE_OUT, seed=0, lr=1e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0,
                 fused_adamw=True, norms=(), dropouts=()):
        self.linears = list(linears)
        for lin in self.linears:
            if lin.bias is not None:
                raise ValueError("DP-SGD-RC here covers bias-free linear layers")
        if estimator not in ("hutch", "hutchpp"):
            raise ValueError(estimator)
        self.C, self.sigma = float(C), float(sigma)
        self.estimator, self.k, self.s, self.r, self.side, self.seed = estimator, k, s, r, side, seed
        self.probe = {"rademacher": D.PROBE_RADEMACHER, "gaussian": D.PROBE_GAUSSIAN}[probe]
        self.master = [lin.weight.detach().t().float().contiguous() for lin in self.linears]
        for lin in self.linears:
            lin.weight.requires_grad_(True)
        self.norms, self.dropouts = list(norms), list(dropouts)
        self._gather_vectors()
        self.hp = dict(lr=lr, beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay)
        self.fused = bool(fused_adamw)
        masters = self.master + ([self.vec_master] if self.norms else [])
        if self.fused:
            self.m = [torch.zeros_like(x) for x in masters]
            self.v = [torch.zeros_like(x) for x in masters]
        else:
            groups = [dict(params=self.master)]
            if self.norms:
                groups.append(dict(params=[self.vec_master], weight_decay=0.0))
            self.opt = torch.optim.AdamW(groups, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay)
        self.steps = 0
        self._A = [None] * len(self.linears)
        self._S = [None] * len(self.linears)
        self._hooks = [lin.register_forward_hook(self._tap(j)) for j, lin in enumerate(self.linears)]
        self._ws_acc = None
        self.last = {}

    def _gather_vectors(self):
        """Lay the norms' parameters side by side: vec_master [1, N] fp32, and for bf16 parameters vec_w [N],
        which the parameters become views of (fp32 ones become views of the master)."""
        params = [q for m in self.norms for q in m.parameters_in_order()]
        self._G, self._sinks = None, []
        if not params:
            return
        if len({q.dtype for q in params}) != 1:
            raise ValueError("the norms' parameters must share a dtype")
        if len({id(q) for q in params}) != len(params):
            raise ValueError("a parameter is listed twice: norms that share parameters cannot be trained")
        flat = torch.cat([q.detach().reshape(-1) for q in params])
        self.vec_master = flat.float().view(1, -1)
        self.vec_w = flat if flat.dtype == torch.bfloat16 else None
        store = self.vec_master.view(-1) if self.vec_w is None else self.vec_w
        at = 0
        for m in self.norms:
            cols = []
            for q in m.parameters_in_order():
                q.data = store[at:at + q.numel()]
                q.requires_grad_(True)
                cols.append(slice(at, at + q.numel()))
                at += q.numel()
            self._sinks.append(self._sink(m, cols))

    def _sink(self, m, cols):
        """What the backward call of norm m writes its per-sample gradients to, during a capture."""
        def rows(B):
            if self._G is None:
                self._G = torch.empty(B, self.vec_master.shape[1], dtype=torch.float32, device=self.vec_master.device)
                self._filled = set()
            if id(m) in self._filled:
                raise RuntimeError("a trained norm ran twice in one step")
            self._filled.add(id(m))
            return self._G[:, cols[0]], self._G[:, cols[1]] if len(cols) > 1 else None
        return rows

    def _tap(self, j):
        def hook(mod, inputs, output):
            self._A[j] = inputs[0]
            self._S[j] = output
        return hook

    def remove_hooks(self):
        for h in self._hooks:
            h.remove()

    def capture(self, loss_fn, key=None):
        """Steps 1-2: per-sample losses [B] and the layers' (A, E) pairs, with the norms' per-sample gradients
        beside them (``Pairs``).  ``key``: that of the dropout masks, by default the step's.  Masks go by the
        row of a call, so micro-batches of one step need a key each."""
        self._G = None
        key = step_seed(self.seed, self.steps) if key is None else key
        try:
            with junction.step_key(key):
                for m, sink in zip(self.norms, self._sinks):
                    m.seed, m.sink = key, sink
                for m in self.dropouts:
                    m.seed = key
                losses = loss_fn()
                if losses.dim() != 1:
                    raise ValueError("loss_fn must return per-sample losses [B]")
                # the norms' weights are listed for the backward pass to reach every norm; their own
                # gradients go to the rows of self._G
                E = torch.autograd.grad(losses.sum(), self._S + [m.weight for m in self.norms],
                                        allow_unused=bool(self.norms))
        finally:
            for m in self.norms:
                m.sink = None
        if self.norms:
            E = E[:len(self._S)]
            if any(e is None for e in E) or self._G is None or len(self._filled) < len(self.norms):
                raise RuntimeError("a trained layer or norm has no part in the loss")
            if any(e.shape[0] != self._G.shape[0] for e in E):
                raise RuntimeError(f"the norms saw a batch of {self._G.shape[0]} samples, the layers another")
        # token-row layouts for the library (no copy when already so; layers fed the
        # same activations keep one pointer, so they share a pass over A)
        pairs = Pairs(((_rows(self._A[j].detach()), _rows(E[j]), j) for j in range(len(self.linears))), self._G)
        self._A = [None] * len(self.linears)
        self._S = [None] * len(self.linears)
        return losses.detach(), pairs

    @staticmethod
    def _vectors(pairs):
        """The norms' per-sample gradients that were captured with these layers."""
        G = getattr(pairs, "vectors", None)
        if G is None:
            raise ValueError("pairs must be what capture returned, the norms' per-sample gradients with the layers'")
        if any(A.shape[0] != G.shape[0] for (A, _, _) in pairs):
            raise ValueError(f"the norms' batch of {G.shape[0]} samples is not the layers'")
        return G

    def estimate(self, pairs, key):
        """Steps 3-4: n2 [B] and c [B]."""
        n2 = D.dprc_norm_vectors(self._vectors(pairs)) if self.norms else None
        more = n2 is not None
        if self.estimator == "hutch":
            return D.dprc_norm_hutch_clip(pairs, self.k, key, self.C, side=self.side, probe=self.probe, n2=n2,
                                          accumulate=more)
        n2 = D.dprc_norm_hutchpp(pairs, self.s, self.r, key, side=self.side, n2=n2, accumulate=more)
        return n2, D.dprc_clip_scale(n2, self.C)

    def private_grads(self, pairs, key, noise=True):
        """Steps 3-6: n2 [B], c [B] and the clipped gradients ([d, p] fp32 per layer, then [1, N] of
        the norms if any are trained), with the noise added unless ``noise`` is false."""
        n2, c = self.estimate(pairs, key)
        grads = self.clipped_sums(pairs, c)
        if noise and self.sigma > 0:
            for j, g in zip([j for (_, _, j) in pairs] + [len(self.linears)], grads):
                D.dprc_add_noise(g, self.sigma, self.C, key, j)
        return n2, c, grads

    def clipped_sums(self, pairs, c):
        """Step 5 for every layer: one call when all are bf16 (the small layers share
        launches), else one call per layer; then for the norms."""
        G = self._vectors(pairs) if self.norms else None
        if all(A.dtype == torch.bfloat16 and E.dtype == torch.bfloat16 for (A, E, _) in pairs):
            grads = D.dprc_clip_accumulate_layers(pairs, c)
        else:
            need = max(D.dprc_clip_accumulate_workspace(A, E) for (A, E, _) in pairs)
            if self._ws_acc is None or self._ws_acc.numel() < need:
                self._ws_acc = torch.empty(max(need, 1), dtype=torch.uint8, device=c.device)
            grads = [D.dprc_clip_accumulate(A, E, c, ws=self._ws_acc) for (A, E, _) in pairs]
        if self.norms:
            grads.append(D.dprc_clip_accumulate_vectors(G, c).view(1, -1))
            if G is self._G:                # from here on only `pairs` holds them
                self._G = None
        return grads

    def update(self, clipped, batch, key):
        """Steps 6-7 fused: per layer, noise + 1/batch + AdamW + bf16 weight write in one pass."""
        t = self.steps + 1
        for j, (lin, th, G) in enumerate(zip(self.linears, self.master, clipped)):
            D.dprc_private_adamw(th, self.m[j], self.v[j], G, self.sigma, self.C, key, j, 1.0 / batch,
                                 step=t, w=lin.weight.detach(), **self.hp)
            lin.weight.grad = None
        if self.norms:
            j = len(self.linears)
            D.dprc_private_adamw(self.vec_master, self.m[j], self.v[j], clipped[j], self.sigma, self.C, key, j,
                                 1.0 / batch, step=t, w=None if self.vec_w is None else self.vec_w.view(-1, 1),
                                 **dict(self.hp, weight_decay=0.0))
        self.steps = t

    def apply(self, grads, batch):
        """Step 7 with torch's AdamW (noisy grads / batch), then refresh the model weights."""
        for m, g in zip(self.master + ([self.vec_master] if self.norms else []), grads):
            m.grad = g.div_(batch)
        self.opt.step()
        with torch.no_grad():
            for lin, m in zip(self.linears, self.master):
                lin.weight.copy_(m.t())
                lin.weight.grad = None
            if self.norms and self.vec_w is not None:
                self.vec_w.copy_(self.vec_master[0])
        self.opt.zero_grad(set_to_none=True)
        self.steps += 1

    def step(self, loss_fn):
        """One full step; returns the per-sample losses (before the update)."""
        losses, pairs = self.capture(loss_fn)
        key = step_seed(self.seed, self.steps)
        n2, c, grads = self.private_grads(pairs, key, noise=not self.fused)
        del pairs
        if self.fused:
            self.update(grads, losses.numel(), key)
        else:
            self.apply(grads, losses.numel())
        self.last = {"n2": n2, "c": c}
        return losses
