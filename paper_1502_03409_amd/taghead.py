"""A head that learns the users' tags (Sec. 2: the data set's other half) from the features the layers have learned.

    features [N, D] -> gated hidden layer [N, F] -> scores of V tags -> softmax cross entropy
    gradients of all three weight matrices -> clipped by their common norm -> one step of gradient descent

The features are those of a trained, frozen layer (`features`: forward pass, pooling, contrast normalisation, in fp32; a head
of bf16 weights takes them cast to bf16), so no gradient reaches them.  What a head answers is a loss (`evaluate`: of one tag an image,
row by row) or what it believes (`answer`: log probabilities of an image's tags, the likeliest tags and their log probabilities, the
entropy).  Images with several tags, or with a reward for what was answered, are learned from through the log probabilities
(`answer` with gradients to come, then `gradients_of`).  A step goes against the gradients, or, with a momentum, along its
orthogonalised form.  `CompressedHead` scores images with weights of 8 bits.

All memory is allocated when the head is made, for a largest batch; a step only enqueues work on the current
stream.  ``python -m paper_1502_03409_amd.taghead`` trains one on synthetic images and prints its cost and how often its likeliest tag is
the image's.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as lc
from . import head as H


class TagHead:
    def __init__(self, D: int, F: int, V: int, batch: int, *, dtype: torch.dtype = torch.float32, act: int = H.LC_ACT_SILU,
                 max_norm: float = 1.0, seed: int = 0, device="cuda", momentum: Optional[float] = None, tags: int = 1, likeliest: int = 0):
        """``momentum``: of orthogonalised steps, None for plain ones.  ``tags``, ``likeliest``: the most tags an image that `answer` is given
        and asked for."""
        self.D, self.F, self.V, self.act, self.max_norm = D, F, V, act, max_norm
        self.code = lc.LC_BF16 if dtype == torch.bfloat16 else lc.LC_F32
        gen = torch.Generator().manual_seed(seed)

        def weights(rows, cols):
            return (torch.randn(rows, cols, generator=gen) * cols ** -0.5).to(dtype).to(device)

        self.wg, self.wu, self.wv = weights(F, D), weights(F, D), weights(V, F)
        self.params = [self.wg, self.wu, self.wv]
        self.grads = [torch.empty_like(w) for w in self.params]
        self.h, self.dh = (torch.empty(batch, F, dtype=dtype, device=device) for _ in range(2))
        self.gu = torch.empty(batch, 2, F, dtype=dtype, device=device)
        self.loss = torch.empty(batch, device=device)
        self.cost, self.norm = torch.empty(1, device=device), torch.empty(1, device=device)
        self.momentum = momentum
        self.momenta = [torch.zeros(w.shape, device=device) for w in self.params] if momentum is not None else []
        # one after the other for each row: a batch's part of each is contiguous, whatever its number of rows and tags
        self.logp, self.top_logp = (torch.empty(batch * k, device=device) for k in (tags, likeliest))
        self.top = torch.empty(batch * likeliest, dtype=torch.int64, device=device)
        self.entropy, self.state = torch.empty(batch, device=device), torch.empty(batch, 3, device=device)
        need = max(H.glu_workspace_bytes(batch, D, F, self.code, True), H.xent_workspace_bytes(batch, F, V, self.code, True),
                   H.grad_clip_workspace_bytes(self.grads), *(H.logp_workspace_bytes(batch, F, V, t, likeliest, self.code, True) for t in (0, tags)),
                   *(H.muon_workspace_bytes(1, *w.shape, self.code) for w in self.params if momentum is not None))
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)
        self.learning = None   # images and tags an image of the answer that gradients_of may follow

    def gradients(self, x: torch.Tensor, target: torch.Tensor) -> None:
        """Cost, loss of every row and gradients of a batch (targets below 0: rows without a tag)."""
        self.learning = None
        n = x.shape[0]
        h, gu, dh = self.h[:n], self.gu[:n], self.dh[:n]
        H.glu_fwd(x, self.wg, self.wu, h, gu, self.act, self.code, self.ws)
        H.xent_fwd_bwd(h, self.wv, target, None, self.loss[:n], self.cost, dh, self.grads[2], self.code, self.ws)
        H.glu_bwd(x, self.wg, self.wu, gu, dh, None, self.grads[0], self.grads[1], self.act, self.code, self.ws)

    def step(self, x: torch.Tensor, target: torch.Tensor, lr: float) -> None:
        """One training step; the cost from before it and the gradients' norm are in ``cost`` and ``norm``."""
        self.gradients(x, target)
        self.update(lr)

    def update(self, lr: float) -> None:
        """Clips the gradients that are there and steps.  With a momentum each value moves by about 0.2 ``lr``, whatever its matrix's sides."""
        self.learning = None
        H.grad_clip(self.grads, None, self.max_norm, self.norm, self.ws)
        if self.momentum is None:
            for w, g in zip(self.params, self.grads):
                w.add_(g, alpha=-lr)
            return
        for w, g, m in zip(self.params, self.grads, self.momenta):
            H.muon_step(w, g, m, None, None, 0.2 * lr * max(w.shape) ** 0.5, 0.0, self.momentum, dtype=self.code, ws=self.ws)

    def answer(self, x: torch.Tensor, tags: Optional[torch.Tensor] = None, likeliest: int = 0, learn: bool = False):
        """What the head says of a batch: log probabilities of ``tags`` [n, T] (below 0: none; rows without any are masked) or None,
        the ``likeliest`` tags and their log probabilities or None, and the entropies.  The results are the head's own buffers.  ``learn``:
        `gradients_of` follows."""
        n, T, K = x.shape[0], 0 if tags is None else tags.shape[1], likeliest
        h, self.learning = self.h[:n], None
        if n * T > self.logp.numel() or n * K > self.top.numel():
            raise ValueError(f"the head was made for fewer tags than {T} given and {K} likeliest ones of {n} images")
        logp = self.logp[:n * T].view(n, T) if T else None
        top, top_logp = (self.top[:n * K].view(n, K), self.top_logp[:n * K].view(n, K)) if K else (None, None)
        H.glu_fwd(x, self.wg, self.wu, h, self.gu[:n] if learn else None, self.act, self.code, self.ws)
        H.logp_fwd(h, self.wv, tags if T else None, logp, self.entropy[:n], top, top_logp, self.state[:n] if learn else None, self.code, self.ws)
        self.learning = (n, T) if learn else None
        return logp, top, top_logp, self.entropy[:n]

    def gradients_of(self, x: torch.Tensor, tags: Optional[torch.Tensor], dlogp: Optional[torch.Tensor], dentropy: Optional[torch.Tensor] = None) -> None:
        """Gradients for given ones of the log probabilities [n, T] and entropies [n] of the batch and tags that `answer` saw last, with ``learn`` and
        the weights as they are: nothing else that computes with the head may lie between."""
        n, T = x.shape[0], 0 if tags is None else tags.shape[1]
        if self.learning != (n, T):
            raise ValueError(f"gradients of {T} tags each of {n} images follow their answer with learn=True, without another call between")
        h, gu, dh = self.h[:n], self.gu[:n], self.dh[:n]
        H.logp_bwd(h, self.wv, tags if T else None, self.logp[:n * T].view(n, T) if T else None, self.state[:n], dlogp, dentropy, dh, self.grads[2],
                   self.code, self.ws)
        H.glu_bwd(x, self.wg, self.wu, gu, dh, None, self.grads[0], self.grads[1], self.act, self.code, self.ws)

    def evaluate(self, x: torch.Tensor, target: torch.Tensor) -> None:
        """Cost and loss of every row, nothing else."""
        self.learning = None
        n = x.shape[0]
        H.glu_fwd(x, self.wg, self.wu, self.h[:n], None, self.act, self.code, self.ws)
        H.xent_fwd(self.h[:n], self.wv, target, None, self.loss[:n], self.cost, self.code, self.ws)


class CompressedHead:
    """A trained head with weights of 8 bits: a quarter (fp32) or half (bf16) of the bytes that an answer waits for."""

    def __init__(self, head: TagHead, batch: int):
        self.act, self.code, dev = head.act, head.code, head.wg.device
        self.V = head.V
        dtype = head.wg.dtype

        def eight_bits(w):
            q = torch.empty(w.shape[0], H.q8_row_bytes(w.shape[1]), dtype=torch.int8, device=dev)
            scale = torch.empty(w.shape[0], device=dev)
            H.q8_rows(w, q, scale, self.code)
            return q, scale

        (self.qg, self.sg), (self.qu, self.su), (self.qv, self.sv) = map(eight_bits, head.params)
        self.h = torch.empty(batch, head.F, dtype=dtype, device=dev)
        self.out = torch.empty(batch, head.V, dtype=dtype, device=dev)
        need = max(H.q8_workspace_bytes(batch, head.D, head.F, self.code), H.q8_workspace_bytes(batch, head.F, head.V, self.code))
        self.ws = torch.empty(need, dtype=torch.uint8, device=dev)

    def scores(self, x: torch.Tensor) -> torch.Tensor:
        """Scores [n, V] of a batch, in the head's own buffer."""
        n = x.shape[0]
        h, out = self.h[:n], self.out[:n]
        H.q8_glu_fwd(x, self.qg, self.sg, self.qu, self.su, h, self.act, self.code, self.ws)
        H.q8_matmul(h, self.qv, self.sv, out, self.code, self.ws)
        return out


def features(g: lc.LcGeom, x: torch.Tensor, w: torch.Tensor, pool=(3, 1, 1e-6), norm=(5, 1.0, 1e-4)) -> torch.Tensor:
    """Pooled and normalised responses of a layer, one row an image."""
    LH, LW, _ = lc.geom_derive(g)
    Hp, Wp = (LH - pool[0]) // pool[1] + 1, (LW - pool[0]) // pool[1] + 1
    y = torch.empty(g.B, LH, LW, g.F, device=x.device)
    p, n = (torch.empty(g.B, Hp, Wp, g.F, device=x.device) for _ in range(2))
    mu, rstd = (torch.empty(g.B, Hp, Wp, device=x.device) for _ in range(2))
    need = lc.workspace_bytes(g, lc.LC_OP_FORWARD)
    lc.lc_forward(g, x, w, None, 1.0, y, lc.LC_F32, torch.empty(need, dtype=torch.uint8, device=x.device) if need else None)
    lc.l2pool_lcn_fwd(y, p, n, mu, rstd, *pool, *norm)
    return n.view(g.B, -1)


def main() -> None:
    """Images of a few kinds, each kind with its own tag and every tenth image without one."""
    gen = torch.Generator().manual_seed(0)
    g = lc.geom(192, 32, 32, 3, 8, 4, 16)
    kinds, vocabulary = 12, 1000
    LH, LW, K = lc.geom_derive(g)
    w = (torch.randn(LH, LW, K, g.F, generator=gen) * K ** -0.5).cuda()
    base = torch.randn(kinds, g.H, g.W, g.C, generator=gen)
    tag = torch.randint(0, vocabulary, (kinds,), generator=gen)
    head = None
    for step in range(60):
        kind = torch.randint(0, kinds, (g.B,), generator=gen)
        x = (base[kind] + torch.randn(g.B, g.H, g.W, g.C, generator=gen)).cuda()
        target = tag[kind]
        target[::10] = -1
        f = features(g, x, w)
        if head is None:
            head = TagHead(f.shape[1], 256, vocabulary, g.B, likeliest=1)
        head.step(f, target.cuda(), lr=0.5)
        if step % 10 == 0 or step == 59:
            right = (head.answer(f, likeliest=1)[1][:, 0].cpu() == tag[kind]).float().mean().item()
            print(f"step {step}: cost {head.cost.item():.4f}, norm of the gradients {head.norm.item():.4f}, likeliest tag right {right:.0%}", flush=True)


if __name__ == "__main__":
    main()
