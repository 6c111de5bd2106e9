"""A head that learns the users' tags (Sec. 2: the data set's other half) from the features the layers have learned.

    features [N, D] -> gated hidden layer [N, F] -> scores of V tags -> softmax cross entropy
    gradients of all three weight matrices -> clipped by their common norm -> one step of gradient descent

The features are those of a trained, frozen layer (`features`: forward pass, pooling, contrast normalisation, in fp32; a head
of bf16 weights takes them cast to bf16), so no gradient reaches them.  What a head answers is a loss: of the tags given to
`evaluate`, row by row.  All memory is allocated when the head is made, for a largest batch; a step only enqueues work on the current
stream.  ``python -m paper_1502_03409_amd.taghead`` trains one on synthetic images and prints its cost.
"""
from __future__ import annotations

import torch

from . import binding as lc
from . import head as H


class TagHead:
    def __init__(self, D: int, F: int, V: int, batch: int, *, dtype: torch.dtype = torch.float32, act: int = H.LC_ACT_SILU,
                 max_norm: float = 1.0, seed: int = 0, device="cuda"):
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
        need = max(H.glu_workspace_bytes(batch, D, F, self.code, True), H.xent_workspace_bytes(batch, F, V, self.code, True),
                   H.grad_clip_workspace_bytes(self.grads))
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)

    def gradients(self, x: torch.Tensor, target: torch.Tensor) -> None:
        """Cost, loss of every row and gradients of a batch (targets below 0: rows without a tag)."""
        n = x.shape[0]
        h, gu, dh = self.h[:n], self.gu[:n], self.dh[:n]
        H.glu_fwd(x, self.wg, self.wu, h, gu, self.act, self.code, self.ws)
        H.xent_fwd_bwd(h, self.wv, target, None, self.loss[:n], self.cost, dh, self.grads[2], self.code, self.ws)
        H.glu_bwd(x, self.wg, self.wu, gu, dh, None, self.grads[0], self.grads[1], self.act, self.code, self.ws)

    def step(self, x: torch.Tensor, target: torch.Tensor, lr: float) -> None:
        """One training step; the cost from before it and the gradients' norm are in ``cost`` and ``norm``."""
        self.gradients(x, target)
        H.grad_clip(self.grads, None, self.max_norm, self.norm, self.ws)
        for w, g in zip(self.params, self.grads):
            w.add_(g, alpha=-lr)

    def evaluate(self, x: torch.Tensor, target: torch.Tensor) -> None:
        """Cost and loss of every row, nothing else."""
        n = x.shape[0]
        H.glu_fwd(x, self.wg, self.wu, self.h[:n], None, self.act, self.code, self.ws)
        H.xent_fwd(self.h[:n], self.wv, target, None, self.loss[:n], self.cost, self.code, self.ws)


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
            head = TagHead(f.shape[1], 256, vocabulary, g.B)
        head.step(f, target.cuda(), lr=0.5)
        if step % 10 == 0 or step == 59:
            print(f"step {step}: cost {head.cost.item():.4f}, norm of the gradients {head.norm.item():.4f}", flush=True)


if __name__ == "__main__":
    main()
