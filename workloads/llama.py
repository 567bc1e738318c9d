"""A Llama-3.2-1B-shaped decoder stack with seeded random weights.

It is the synthetic model of the end-to-end DP-SGD-RC step (no trained weights
or datasets are available): token embedding, ``layers`` blocks of RMSNorm ->
grouped-query attention with rotary positions -> residual, RMSNorm -> SwiGLU
MLP -> residual, a final RMSNorm and an untied lm_head.  Every projection is a
bias-free ``nn.Linear``.  Default sizes are Llama-3.2-1B's: hidden 2048, MLP
8192, 32 query heads and 8 key/value heads of width 64, vocabulary 128256, 16
blocks, rotary base 500000.

Attention scores, softmax and the value product run in fp32 on contiguous
operands; the projections run in the weights' dtype (bf16 by default).  q, k
and v read the same normed activations, as do gate and up.

With ``junctions`` the norms, the residual sums before them and a dropout of rate
``dropout`` on every branch run as ``paper_2605_24879_amd.junction.Junction``
(``norm``: "rms" or "layer"), which ``norms()`` lists for private training, and a
dropout of the same rate inside the MLP as ``junction.Dropout`` (``dropouts()``).

With ``rotary`` the rotary positions run as ``paper_2605_24879_amd.rotary.Rotary``, which turns q and k in one call;
with ``head`` the output layer and its cross entropy as ``paper_2605_24879_amd.head.Head``: the model called with targets
then gives per-token losses and stores no logits, and ``head`` is what private training takes.

``linears()`` lists the projections in model order (per block q, k, v, o,
gate, up, down; then lm_head, unless it runs as ``head``), which keeps the shared-input layers adjacent.
"""

import itertools
import math

import torch
import torch.nn as nn
import torch.nn.functional as F

LLAMA_3_2_1B = dict(layers=16, hidden=2048, mlp=8192, heads=32, kv_heads=8, vocab=128256, rope_base=500000.0)


class RMSNorm(nn.Module):
    def __init__(self, n, eps=1e-5):
        super().__init__()
        self.weight = nn.Parameter(torch.ones(n))
        self.eps = eps

    def forward(self, x):
        xf = x.float()
        y = xf * torch.rsqrt(xf.pow(2).mean(-1, keepdim=True) + self.eps)
        return (y * self.weight.float()).to(x.dtype)


def _rope_tables(T, hd, base, device):
    inv = 1.0 / (base ** (torch.arange(0, hd, 2, device=device, dtype=torch.float32) / hd))
    ang = torch.arange(T, device=device, dtype=torch.float32)[:, None] * inv[None, :]
    return torch.cos(ang), torch.sin(ang)


def _rope(x, cos, sin):
    # x: [B, H, T, hd] fp32; rotate the (first half, second half) pairs
    h = x.shape[-1] // 2
    x1, x2 = x[..., :h], x[..., h:]
    return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1)


class Block(nn.Module):
    def __init__(self, hidden, mlp, heads, kv_heads, make_norm=RMSNorm, make_drop=nn.Identity, rotary=None):
        super().__init__()
        hd = hidden // heads
        self.heads, self.kv_heads, self.hd = heads, kv_heads, hd
        self.norm1 = make_norm(hidden)
        self.q = nn.Linear(hidden, heads * hd, bias=False)
        self.k = nn.Linear(hidden, kv_heads * hd, bias=False)
        self.v = nn.Linear(hidden, kv_heads * hd, bias=False)
        self.o = nn.Linear(heads * hd, hidden, bias=False)
        self.norm2 = make_norm(hidden)
        self.gate = nn.Linear(hidden, mlp, bias=False)
        self.up = nn.Linear(hidden, mlp, bias=False)
        self.down = nn.Linear(mlp, hidden, bias=False)
        self.act_drop = make_drop()
        self.rotary = rotary                   # None: _rope

    def attend(self, h, cos, sin, mask):
        B, T, _ = h.shape
        q = self.q(h).view(B, T, self.heads, self.hd)
        k = self.k(h).view(B, T, self.kv_heads, self.hd)
        v = self.v(h).view(B, T, self.kv_heads, self.hd).transpose(1, 2).float()
        if self.rotary is not None:
            q, k = (x.transpose(1, 2) for x in self.rotary(q, k, heads_first=True, out_dtype=torch.float32))
        else:
            q, k = (_rope(x.transpose(1, 2).float(), cos, sin) for x in (q, k))
        rep = self.heads // self.kv_heads
        k = k.repeat_interleave(rep, dim=1)
        v = v.repeat_interleave(rep, dim=1).contiguous()
        s = torch.matmul(q.contiguous(), k.transpose(-1, -2).contiguous()) * (1.0 / math.sqrt(self.hd))
        p = torch.softmax(s + mask, dim=-1)
        a = torch.matmul(p, v).transpose(1, 2).reshape(B, T, self.heads * self.hd).to(h.dtype)
        return self.o(a)

    def feed(self, h):
        return self.down(self.act_drop(F.silu(self.gate(h)) * self.up(h)))

    def forward(self, x, cos, sin, mask):
        x = x + self.attend(self.norm1(x), cos, sin, mask)
        return x + self.feed(self.norm2(x))


class JunctionBlock(Block):
    """The block with each residual sum in the junction before the next norm: from a branch not yet added
    and the residual (None before the first sum) to the next such pair."""

    def forward(self, branch, x, cos, sin, mask):
        h, x = self.norm1(branch, x)
        h, x = self.norm2(self.attend(h, cos, sin, mask), x)
        return self.feed(h), x


class LlamaShaped(nn.Module):
    def __init__(self, layers=16, hidden=2048, mlp=8192, heads=32, kv_heads=8, vocab=128256,
                 rope_base=500000.0, junctions=False, norm="rms", dropout=0.0, rotary=False, head=False):
        super().__init__()
        self.embed = nn.Embedding(vocab, hidden)
        self.junctions = bool(junctions)
        make_norm, make_drop, block = RMSNorm, nn.Identity, Block
        if self.junctions:
            from paper_2605_24879_amd.junction import Dropout, Junction
            sites = itertools.count()
            make_norm, block = lambda n: Junction(n, kind=norm, p=dropout, site_id=next(sites)), JunctionBlock
            make_drop = lambda: Dropout(dropout, site_id=next(sites))
        elif norm != "rms" or dropout:
            raise ValueError("layer norm and dropout come with junctions")
        rot = None
        if rotary:
            from paper_2605_24879_amd.rotary import Rotary
            with torch.device("cpu"):           # frequencies are values, whatever device the model is laid out on
                rot = Rotary(hidden // heads, base=rope_base)
        self.blocks = nn.ModuleList([block(hidden, mlp, heads, kv_heads, make_norm, make_drop, rot) for _ in range(layers)])
        self.tables = rot is None
        self.norm = make_norm(hidden)
        self.lm_head = nn.Linear(hidden, vocab, bias=False)
        head_of = None
        if head:
            from paper_2605_24879_amd.head import Head
            head_of = Head(self.lm_head)
        self.__dict__["head"] = head_of         # not a submodule: the weight keeps its one name
        self.rope_base = rope_base
        self.hd = hidden // heads

    def linears(self):
        out = []
        for b in self.blocks:
            out += [b.q, b.k, b.v, b.o, b.gate, b.up, b.down]
        return out if self.head is not None else out + [self.lm_head]

    def norms(self):
        return [m for b in self.blocks for m in (b.norm1, b.norm2)] + [self.norm]

    def dropouts(self):
        return [b.act_drop for b in self.blocks] if self.junctions else []

    def forward(self, tokens, targets=None):
        """Logits [B, T, vocab], or with targets [B, T] (and the model's ``head``) the tokens' losses [B, T]."""
        if targets is not None and self.head is None:
            raise ValueError("losses come with head=True")
        B, T = tokens.shape
        cos, sin = _rope_tables(T, self.hd, self.rope_base, tokens.device) if self.tables else (None, None)
        mask = torch.full((T, T), float("-inf"), device=tokens.device).triu(1)
        x = self.embed(tokens)
        if self.junctions:
            branch, x = x, None
            for b in self.blocks:
                branch, x = b(branch, x, cos, sin, mask)
            y = self.norm(branch, x)[0]
        else:
            for b in self.blocks:
                x = b(x, cos, sin, mask)
            y = self.norm(x)
        return self.lm_head(y) if targets is None else self.head(y, targets)


def build(seed=0, device="cuda", dtype=torch.bfloat16, **sizes):
    """A seeded LlamaShaped model (weights ~ N(0, 0.02^2), norms 1) in ``dtype``."""
    cfg = dict(LLAMA_3_2_1B)
    cfg.update(sizes)
    g = torch.Generator(device=device).manual_seed(seed)
    with torch.device("meta"):
        model = LlamaShaped(**cfg)
    model = model.to_empty(device=device)
    with torch.no_grad():
        for name, prm in model.named_parameters():
            if prm.dim() == 2:
                prm.normal_(0.0, 0.02, generator=g)
            else:
                prm.fill_(0.0 if name.endswith("bias") else 1.0)
    return model.to(dtype)


def tokens(B, T, vocab, seed=0, device="cuda"):
    """Seeded token ids [B, T + 1] (inputs are [:, :-1], next-token targets [:, 1:])."""
    g = torch.Generator(device=device).manual_seed(seed + 1)
    return torch.randint(0, vocab, (B, T + 1), generator=g, device=device)


def per_sample_loss(logits, targets):
    """Mean next-token cross-entropy of each sample (fp32): [B]."""
    B, T, V = logits.shape
    ce = F.cross_entropy(logits.float().reshape(B * T, V), targets.reshape(B * T), reduction="none")
    return ce.view(B, T).mean(dim=1)
