"""Skip-gram with the full softmax: the objective that negative sampling approximates.

A pair (src, ctx) is scored against every row of the context table instead of a few sampled ones:
loss = -log softmax(context . vertex[src])[ctx].  A step looks up the batch's vertex rows, takes the softmax cross
entropy against the whole context table without keeping the scores, brings the gradients back to both tables (the
vertex table's by sorted ids) and moves both with AdamW, or with Muon, whose updates have singular values near 1.  With an entropy weight the
objective also holds up the entropy of what the model answers.  predict() answers with it: the most probable contexts of given nodes.  Every part is a call
of the library; torch allocates and marks the pairs that are left out.
"""
from __future__ import annotations

import math

import torch

import paper_2005_13789_amd as ne


class SoftmaxTrainer:
    """Trains vertex and context (float32 [num_nodes][dim], CUDA, updated in place) on batches of at most `batch` pairs.

    compute: torch.float32, or torch.bfloat16 for products and gradients in bf16 on rounded copies of the tables that
    every step of the optimizer writes.  state_bits: 32, or 8 for AdamW states of a byte each.

    optimizer: "adamw", or "muon" (momentum with Nesterov's look ahead, Newton-Schulz updates of each table as one matrix, scaled to elements as
    large as AdamW's: learning rates are comparable).  entropy_weight: what is minimised is loss - entropy_weight * entropy."""

    def __init__(self, vertex: torch.Tensor, context: torch.Tensor, batch: int, state_bits: int = 32, weight_decay: float = 0.0,
                 compute: torch.dtype = torch.float32, seed: int = 0, optimizer: str = "adamw", momentum: float = 0.95,
                 entropy_weight: float = 0.0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        if vertex.shape != context.shape or vertex.dim() != 2:
            raise ValueError("vertex and context must both be [num_nodes][dim]")
        if optimizer not in ("adamw", "muon") or (optimizer == "muon" and state_bits != 32):
            raise ValueError("optimizer must be 'adamw', or 'muon' with state_bits 32")
        if optimizer == "muon" and min(vertex.shape) > ne.NE_ORTHOGONAL_MAX_SIDE:
            raise ValueError(f"Muon takes tables whose smaller side is at most {ne.NE_ORTHOGONAL_MAX_SIDE}")
        if not math.isfinite(entropy_weight):
            raise ValueError("entropy_weight must be finite")
        mu, decay = torch.tensor([momentum, weight_decay], dtype=torch.float32).tolist()       # as the step takes them
        if optimizer == "muon" and not (0.0 <= mu < 1.0 and 0.0 <= decay < math.inf):
            raise ValueError("Muon takes a momentum of 0 to 1, 1 excluded, and a finite weight_decay >= 0")
        V, d = vertex.shape
        dev = vertex.device
        self.entropy_weight, self.momentum, self.weight_decay = entropy_weight, momentum, weight_decay
        self.batch, self.steps = batch, 0
        self.tables = [vertex, context]
        copies = None
        if compute == torch.bfloat16:
            copies = [t.bfloat16() for t in self.tables]
        self.rows = copies if copies is not None else self.tables       # what products read
        self.grads = [torch.empty((V, d), dtype=compute, device=dev) for _ in range(2)]
        self.h, self.dh = (torch.empty((batch, d), dtype=compute, device=dev) for _ in range(2))
        self.loss, self.lse = (torch.empty(batch, dtype=torch.float32, device=dev) for _ in range(2))
        size = max(ne.ne_embed_workspace_bytes(V, d, batch), ne.ne_xent_workspace_bytes(batch, V, d, compute, False),
                   ne.ne_xent_workspace_bytes(batch, V, d, compute, True))
        if entropy_weight:
            self.entropy = torch.empty(batch, dtype=torch.float32, device=dev)
            size = max(size, ne.ne_logprob_workspace_bytes(batch, V, d, compute), ne.ne_logprob_workspace_bytes(batch, V, d, compute, grad=True))
        if optimizer == "muon":
            size = max(size, ne.ne_orthogonalize_workspace_bytes(V, d))
        self.work = torch.empty(size, dtype=torch.uint8, device=dev)     # one after the other on one stream: shared by the calls
        self.opt, self.copies = None, copies
        if optimizer == "muon":
            self.momenta = [torch.zeros((V, d), device=dev) for _ in range(2)]
            return
        kw = {}
        if state_bits == 8:
            states = [[torch.zeros((V, d), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2)] for _ in range(2)]
            blocks = -(-V * d // ne.NE_ADAMW_BLOCK)
            kw["m_scale"], kw["v_scale"] = ([torch.zeros(blocks, device=dev) for _ in range(2)] for _ in range(2))
        else:
            states = [[torch.zeros((V, d), device=dev) for _ in range(2)] for _ in range(2)]
        opt_work = torch.empty(ne.ne_adamw_workspace_bytes([V * d] * 2), dtype=torch.uint8, device=dev)
        self.opt = ne.ne_create_adamw(self.tables, self.grads, *states, opt_work, weight_decay=weight_decay, params_bf16=copies, seed=seed, **kw)

    def step(self, pairs: torch.Tensor, lr: float) -> torch.Tensor:
        """One step of the pairs' summed loss / n, pairs int32 [n][2] (CUDA, n <= batch).  A pair of which either id is outside the
        tables (walks are padded with -1) is left out: its loss is 0 and it adds nothing to the gradients; n is the number of all pairs, so that
        one of them weighs the same whatever else is in the step.  Returns the pairs' losses before the step (a view that the next
        step overwrites)."""
        if pairs.dim() != 2 or pairs.shape[1] != 2:
            raise ValueError("pairs must be [n][2]")
        n = int(pairs.shape[0])
        if n < 1 or n > self.batch:
            raise ValueError(f"a step takes 1 to {self.batch} pairs")
        src = pairs[:, 0].contiguous()
        ctx = torch.where(src.clamp(0, self.tables[0].shape[0] - 1) == src, pairs[:, 1], -1)
        h, dh, loss, lse = self.h[:n], self.dh[:n], self.loss[:n], self.lse[:n]
        ne.ne_embed_lookup(self.rows[0], src, h)
        if self.entropy_weight:
            entropy = self.entropy[:n]
            ne.ne_logprob(h, self.rows[1], ctx, lse, self.work, logp=loss, entropy=entropy)
            ne.ne_logprob_grad(h, self.rows[1], ctx, lse, entropy, dh, self.grads[1], self.work, logp_scale=-1.0 / n, entropy_scale=-self.entropy_weight / n)
            loss.neg_()
        else:
            ne.ne_xent_loss(h, self.rows[1], ctx, loss, lse, self.work)
            ne.ne_xent_grad(h, self.rows[1], ctx, lse, dh, self.grads[1], self.work, scale=1.0 / n)
        ne.ne_embed_grad(src, dh, self.grads[0], self.work)
        self.steps += 1
        if self.opt is not None:
            ne.ne_adamw_step(self.opt, self.steps, lr)
            return loss
        for i, table in enumerate(self.tables):
            ne.ne_muon_step(table, self.grads[i], self.momenta[i], self.work, lr, momentum=self.momentum, weight_decay=self.weight_decay,
                            scale=0.2 * math.sqrt(max(table.shape)), param_bf16=self.copies[i] if self.copies is not None else None)
        return loss

    def predict(self, nodes: torch.Tensor, k: int = 10):
        """The k most probable contexts of nodes int32 [n] (CUDA, n <= batch) at the current tables: (ids int32 [n][k], their log probabilities
        float32 [n][k], the entropies float32 [n]).  A node outside the tables has no answers: -1, minus infinity, 0.
        The workspace is the call's own, of n nodes (ne_logprob_workspace_bytes)."""
        n = int(nodes.numel())
        if n < 1 or n > self.batch:
            raise ValueError(f"answers are given for 1 to {self.batch} nodes at a time")
        if not 1 <= k <= ne.NE_TOP_MAX:
            raise ValueError(f"k must be 1 to {ne.NE_TOP_MAX}")
        V, d = self.tables[0].shape
        dev = self.tables[0].device
        work = torch.empty(ne.ne_logprob_workspace_bytes(n, V, d, self.h.dtype, k=k), dtype=torch.uint8, device=dev)
        h = self.h[:n]
        ne.ne_embed_lookup(self.rows[0], nodes, h)
        ids = torch.empty((n, k), dtype=torch.int32, device=dev)
        logp, lse, entropy = torch.empty((n, k), device=dev), torch.empty(n, device=dev), torch.empty(n, device=dev)
        # (the nodes themselves mark the rows that count)
        ne.ne_logprob(h, self.rows[1], nodes, lse, work, entropy=entropy, top_ids=ids, top_logp=logp)
        return ids, logp, entropy
