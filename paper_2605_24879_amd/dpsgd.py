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

Only the listed linear layers are trained, and the norms and the head given as ``norms`` and ``head``;
every other parameter (embedding, other norms) is held fixed.  Probes, noise
and the masks of every ``junction`` module that the loss runs are keyed by a
per-step seed derived from (seed, step), so they are fresh every step.

With ``norms`` (``junction.Junction`` modules), step 2 goes on through the first
norm; the backward calls write every sample's weight and bias gradients side by
side into one [B, N] matrix, which goes with the layers' pairs; step 3 starts from its rows' exact squared norms
(``dprc_norm_vectors``), step 5 adds its clipped sum
(``dprc_clip_accumulate_vectors``), and steps 6 and 7 treat all of them as one
more layer, without weight decay.

With ``head`` (a ``head.Head``, whose losses the loss function takes), the output layer is trained without
its logits or their gradient ever being stored: the backward call of step 2 goes through the vocabulary in
pieces and estimates the head's part of the squared norms on the way, step 5 goes through it once more for
the clipped sum, and steps 6 and 7 treat its weight as one more layer.

With ``max_norm`` the noisy mean gradient of all layers is clipped to that joint norm between steps 6 and 7
(``dprc_grad_clip``): post-processing, which bounds an update that is mostly noise.
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


class HeadPart:
    """The trained head's part of a capture: what its gradients are formed from with the weights of `state`, and the
    estimates n2 under key."""

    def __init__(self, h, target, lse, g, key, n2, state):
        self.h, self.target, self.lse, self.g, self.key, self.n2, self.state = h, target, lse, g, key, n2, state


class Pairs(list):
    """What a capture gives: (A, E, layer) of every trained layer, in ``vectors`` the per-sample
    gradients [B, N] of the trained norms and in ``head`` the head's part (None where there are none).  Whoever
    makes another list of them for a step with norms or a head hands these on."""

    def __init__(self, items=(), vectors=None, head=None):
        super().__init__(items)
        self.vectors, self.head = vectors, head


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
    ``head``: the ``head.Head`` that gives the losses, if its weight is trained (with "hutch"
    only; for the estimates it counts as layers of ``dprc.HEAD_BLOCK`` outputs each).
    ``max_norm``: of the noisy mean gradient, None for no such clipping.
    """

    def __init__(self, linears, C, sigma, estimator="hutch", k=16, probe="rademacher", s=16, r=32,
                 side=D.SIDE_OUT, seed=0, lr=1e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0,
                 fused_adamw=True, norms=(), dropouts=(), head=None, max_norm=None):
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
        self._head = None
        self.head, self.max_norm = head, None if max_norm is None else float(max_norm)
        if self.max_norm is not None and not 0.0 < self.max_norm < float("inf"):
            raise ValueError("max_norm must be positive and finite")
        if head is not None:
            if estimator != "hutch":
                raise ValueError("a trained head's norms are estimated by hutch")
            if any(lin.weight is head.linear.weight for lin in self.linears):
                raise ValueError("the head's layer is listed among the linears too")
            head.linear.weight.requires_grad_(True)
            self.head_master = head.linear.weight.detach().t().float().contiguous()
        self.hp = dict(lr=lr, beta1=betas[0], beta2=betas[1], eps=eps, weight_decay=weight_decay)
        self.fused = bool(fused_adamw)
        if self.fused:
            self.m = [torch.zeros_like(x) for x in self._masters()]
            self.v = [torch.zeros_like(x) for x in self._masters()]
        else:
            groups = [dict(params=self.master + ([self.head_master] if head is not None else []))]
            if self.norms:
                groups.append(dict(params=[self.vec_master], weight_decay=0.0))
            self.opt = torch.optim.AdamW(groups, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay)
        self.steps = 0
        self._A = [None] * len(self.linears)
        self._S = [None] * len(self.linears)
        self._hooks = [lin.register_forward_hook(self._tap(j)) for j, lin in enumerate(self.linears)]
        self._ws_acc = None
        self.last = {}

    def _masters(self):
        """The fp32 masters in the order of the gradients: the layers, the norms, the head."""
        return self.master + ([self.vec_master] if self.norms else []) + ([self.head_master] if self.head is not None else [])

    def _numbers(self, layers):
        """The numbers that key the noise of the gradients of these layers, the norms and the head."""
        n = len(self.linears)
        return layers + ([n] if self.norms else []) + ([n + 1] if self.head is not None else [])

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

    def _head_args(self, key):
        """How the head's norms are estimated: its blocks are numbered behind the linear layers."""
        return dict(k=self.k, seed=key, layer_id=len(self.linears), side=self.side, probe=self.probe)

    def _head_state(self):
        """What changes with the head's weight, by this step's updates or otherwise."""
        return self.steps, self.head.linear.weight._version

    def _take_head(self, key):
        """What the head's backward call does during a capture: the estimates on the way to dh."""
        self._head = None

        def take(h, weight, target, lse, g, want_h):
            if self._head is not None:
                raise RuntimeError("the trained head ran twice in one step")
            dh, _, n2 = D.dprc_head_backward(h, weight, target, lse, g, hidden_grad=want_h, weight_grad=False,
                                             **self._head_args(key))
            # (a copy of the targets: a caller may fill its buffer anew before the head is read again)
            self._head = HeadPart(h.detach(), target.clone(), lse, g, key, n2, self._head_state())
            return dh
        return take

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
        step = step_seed(self.seed, self.steps)
        key = step if key is None else key
        try:
            with junction.step_key(key):
                for m, sink in zip(self.norms, self._sinks):
                    m.seed, m.sink = key, sink
                for m in self.dropouts:
                    m.seed = key
                if self.head is not None:
                    self.head.sink = self._take_head(step)
                losses = loss_fn()
                if losses.dim() != 1:
                    raise ValueError("loss_fn must return per-sample losses [B]")
                # the norms' weights and the head's are listed for the backward pass to reach every norm and the
                # head; their own gradients go to the rows of self._G and into the head's part
                more = [m.weight for m in self.norms] + ([self.head.linear.weight] if self.head is not None else [])
                E = torch.autograd.grad(losses.sum(), self._S + more, allow_unused=bool(more))
        finally:
            for m in self.norms:
                m.sink = None
            if self.head is not None:
                self.head.sink = None
            part, self._head = self._head, None
        E = E[:len(self._S)]
        if any(e is None for e in E) or (self.norms and (self._G is None or len(self._filled) < len(self.norms))):
            raise RuntimeError("a trained layer or norm has no part in the loss")
        if self.norms and any(e.shape[0] != self._G.shape[0] for e in E):
            raise RuntimeError(f"the norms saw a batch of {self._G.shape[0]} samples, the layers another")
        if self.head is not None:
            if part is None:
                raise RuntimeError("the trained head has no part in the loss")
            if any(x.shape[0] != part.h.shape[0] for x in [losses, *E, *([self._G] if self.norms else [])]):
                raise RuntimeError(f"the head saw a batch of {part.h.shape[0]} samples, the loss or the layers another")
        # token-row layouts for the library (no copy when already so; layers fed the
        # same activations keep one pointer, so they share a pass over A)
        pairs = Pairs(((_rows(self._A[j].detach()), _rows(E[j]), j) for j in range(len(self.linears))), self._G, part)
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

    def _part(self, pairs):
        """The head's part that was captured with these layers."""
        part = getattr(pairs, "head", None)
        if part is None:
            raise ValueError("pairs must be what capture returned, the head's part with the layers'")
        if part.state != self._head_state():
            raise RuntimeError("the head's weight has changed since the capture: its gradients are formed from it again")
        batches = [A.shape[0] for (A, _, _) in pairs] + ([pairs.vectors.shape[0]] if self.norms else [])
        if any(B != part.h.shape[0] for B in batches):
            raise ValueError(f"the head's batch of {part.h.shape[0]} samples is not the layers'")
        return part

    def estimate(self, pairs, key):
        """Steps 3-4: n2 [B] and c [B]."""
        n2 = D.dprc_norm_vectors(self._vectors(pairs)) if self.norms else None
        if self.head is not None:
            part = self._part(pairs)
            own = part.n2
            if part.key != key:                 # captured under another step's key
                own = D.dprc_head_backward(part.h, self.head.linear.weight.detach(), part.target, part.lse, part.g,
                                           hidden_grad=False, weight_grad=False, **self._head_args(key))[2]
            n2 = own.clone() if n2 is None else n2 + own
        more = n2 is not None
        if not pairs and more:                  # no linear layers
            return n2, D.dprc_clip_scale(n2, self.C)
        if self.estimator == "hutch":
            return D.dprc_norm_hutch_clip(pairs, self.k, key, self.C, side=self.side, probe=self.probe, n2=n2,
                                          accumulate=more)
        n2 = D.dprc_norm_hutchpp(pairs, self.s, self.r, key, side=self.side, n2=n2, accumulate=more)
        return n2, D.dprc_clip_scale(n2, self.C)

    def private_grads(self, pairs, key, noise=True):
        """Steps 3-6: n2 [B], c [B] and the clipped gradients ([d, p] fp32 per layer, then [1, N] of
        the norms and [d, V] of the head where these are trained), with the noise added unless ``noise``
        is false."""
        n2, c = self.estimate(pairs, key)
        grads = self.clipped_sums(pairs, c)
        if noise and self.sigma > 0:
            for j, g in zip(self._numbers([j for (_, _, j) in pairs]), grads):
                D.dprc_add_noise(g, self.sigma, self.C, key, j)
        return n2, c, grads

    def clipped_sums(self, pairs, c):
        """Step 5 for every layer: one call when all are bf16 (the small layers share
        launches), else one call per layer; then for the norms and the head."""
        G = self._vectors(pairs) if self.norms else None
        part = self._part(pairs) if self.head is not None else None
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
        if part is not None:
            grads.append(D.dprc_head_clip_accumulate(part.h, self.head.linear.weight.detach(), part.target, part.lse, part.g, c))
        return grads

    def update(self, clipped, batch, key, noise=True):
        """Steps 6-7 fused: per layer, noise (unless ``noise`` is false: it is in them already) + 1/batch + AdamW +
        bf16 weight write in one pass."""
        t, sigma = self.steps + 1, self.sigma if noise else 0.0
        for j, (lin, th, G) in enumerate(zip(self.linears, self.master, clipped)):
            D.dprc_private_adamw(th, self.m[j], self.v[j], G, sigma, self.C, key, j, 1.0 / batch,
                                 step=t, w=lin.weight.detach(), **self.hp)
            lin.weight.grad = None
        if self.norms:
            j = len(self.linears)
            D.dprc_private_adamw(self.vec_master, self.m[j], self.v[j], clipped[j], sigma, self.C, key, j,
                                 1.0 / batch, step=t, w=None if self.vec_w is None else self.vec_w.view(-1, 1),
                                 **dict(self.hp, weight_decay=0.0))
        if self.head is not None:
            lin = self.head.linear
            D.dprc_private_adamw(self.head_master, self.m[-1], self.v[-1], clipped[-1], sigma, self.C, key,
                                 self._numbers([])[-1], 1.0 / batch, step=t, w=lin.weight.detach(), **self.hp)
            lin.weight.grad = None
        self.steps = t

    def apply(self, grads, batch):
        """Step 7 with torch's AdamW (noisy grads / batch), then refresh the model weights."""
        for m, g in zip(self._masters(), grads):
            m.grad = g.div_(batch)
        self.opt.step()
        with torch.no_grad():
            for lin, m in zip(self.linears, self.master):
                lin.weight.copy_(m.t())
                lin.weight.grad = None
            if self.norms and self.vec_w is not None:
                self.vec_w.copy_(self.vec_master[0])
            if self.head is not None:
                self.head.linear.weight.copy_(self.head_master.t())
                self.head.linear.weight.grad = None
        self.opt.zero_grad(set_to_none=True)
        self.steps += 1

    def step(self, loss_fn):
        """One full step; returns the per-sample losses (before the update)."""
        losses, pairs = self.capture(loss_fn)
        key = step_seed(self.seed, self.steps)
        batch, noisy = losses.numel(), not self.fused or self.max_norm is not None
        n2, c, grads = self.private_grads(pairs, key, noise=noisy)
        del pairs
        self.last = {"n2": n2, "c": c}
        if self.max_norm is not None:
            self.last["norm"] = D.dprc_grad_clip(grads, self.max_norm * batch)[1] / batch
        if self.fused:
            self.update(grads, batch, key, noise=not noisy)
        else:
            self.apply(grads, batch)
        return losses
