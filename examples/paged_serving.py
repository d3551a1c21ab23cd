"""Decoding for a batch of requests over a paged cache: the paged calls one after
the other, as a server's step makes them.

A small random model (two layers, grouped queries, a rotary embedding) drafts a
tree for every request, verifies all trees in one pass and keeps the accepted
paths.  Requests begin with prompts of different lengths, end at different
times, and give their pages back.  No length is read on the host inside a step.
With --q4 the cache holds 4 bits an element, and the model norms its heads.

    python examples/paged_serving.py [--q4]     # needs a GPU and the built library
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2606_27550_gb300 as tv  # noqa: E402
from paper_2606_27550_gb300 import synth  # noqa: E402


class Model:
    """Random weights; hidden states flow through attention only."""

    def __init__(self, seed=0, layers=2, q_heads=8, kv_heads=2, head_dim=64, vocab=1000):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers, self.Hq, self.H, self.d, self.vocab = layers, q_heads, kv_heads, head_dim, vocab
        self.width = q_heads * head_dim

        def weight(*shape, std):
            return (std * torch.randn(shape, generator=g, device="cuda")).bfloat16()

        self.embed = weight(vocab, self.width, std=1.0)
        self.qkv = [weight(self.width, self.width + 2 * kv_heads * head_dim, std=self.width ** -0.5) for _ in range(layers)]
        self.out = [weight(self.width, self.width, std=self.width ** -0.5) for _ in range(layers)]
        self.head = weight(self.width, vocab, std=2.0 * self.width ** -0.5)
        self.q_norm, self.k_norm = ([1.0 + weight(head_dim, std=0.1) for _ in range(layers)] for _ in range(2))


class Server:
    """The state of a batch of request slots, and its step; q4: over a cache of 4 bits, heads normed."""

    def __init__(self, model: Model, batch=4, n_pages=256, page_size=16, max_pages=64, softcap=30.0, q4=False):
        self.m, self.B, self.softcap, self.q4 = model, batch, softcap, q4
        dev, i32 = "cuda", torch.int32
        self.bank = tv.Bank(8, torch.cuda.current_device())
        self.parents = [synth.chain(1), synth.rank_product_tree((3, 2, 1), 8), synth.rank_product_tree((4, 3, 2, 1), 26)]
        for p in self.parents:
            self.bank.add(p)
        self.nodes = torch.tensor([len(p) for p in self.parents], dtype=i32, device=dev)
        self.rows = 64 * batch
        self.pool = tv.make_page_pool(n_pages, batch)
        shape = (model.layers, n_pages, model.H, page_size, model.d)
        self.pages = (tv.make_pages_q4(*shape, torch.bfloat16) if q4 else
                      tv.Pages(torch.empty(shape, dtype=torch.bfloat16, device=dev),
                               torch.empty(shape, dtype=torch.bfloat16, device=dev)))
        self.req = tv.Requests(row_start=torch.zeros(batch + 1, dtype=i32, device=dev),
                               tree=torch.full((batch,), -1, dtype=i32, device=dev),
                               lens=torch.zeros(batch, dtype=i32, device=dev),
                               table=torch.zeros((batch, max_pages), dtype=i32, device=dev), page_size=page_size)
        # the same slots while they bring prompts
        self.fill = tv.Requests(row_start=self.req.row_start, lens=self.req.lens, table=self.req.table,
                                page_size=page_size, n_new=torch.zeros(batch, dtype=i32, device=dev))
        self.status = torch.zeros(batch, dtype=i32, device=dev)
        self.plan = tv.make_paged_plan(batch)
        self.ws = tv.make_workspace(tv.tb_workspace_size(0, 1, model.H, model.Hq, model.d, 0))
        self.logit_ws = tv.make_workspace(tv.tb_logits_workspace_size(batch, self.rows, model.vocab))
        self.results = tv.make_results(batch)
        self.history = torch.zeros((batch, max_pages * page_size), dtype=i32, device=dev)
        self.said = torch.zeros(batch, dtype=i32, device=dev)   # tokens of the history
        self.asked = torch.zeros(batch, dtype=i32, device=dev)  # of them the prompt's
        self.penalty = torch.full((batch,), 1.2, device=dev)
        self.presence = torch.full((batch,), 0.1, device=dev)

    def _slots(self, rows):
        return (torch.empty(rows, dtype=torch.int64, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"))

    def _layer(self, layer, x, slots, positions, attend):
        m, rows = self.m, x.shape[0]
        qkv = (x @ m.qkv[layer]).view(rows, m.Hq + 2 * m.H, m.d)
        q = torch.empty((rows, m.Hq, m.d), dtype=x.dtype, device="cuda")
        args = dict(layer=layer, q=qkv[:, :m.Hq], q_out=q, positions=positions, rope_theta=10000.0)
        k, v = qkv[:, m.Hq:m.Hq + m.H], qkv[:, m.Hq + m.H:]
        if self.q4:
            tv.paged_kv_store_q4(self.pages, slots, k, v, q_norm=m.q_norm[layer], k_norm=m.k_norm[layer], **args)
        else:
            tv.paged_kv_store(self.pages, slots, k, v, **args)
        if not attend:
            return x
        out = torch.zeros_like(q)
        attention = tv.paged_tree_attention_q4 if self.q4 else tv.paged_tree_attention
        attention(self.bank, self.req, self.pages, self.plan, q, out, self.ws, layer=layer, softcap=self.softcap)
        return x + out.view(rows, m.width) @ m.out[layer]

    def admit(self, prompts):
        """Prompts (token lists, by slot): their keys and values into pages.  (The toy model's layers see
        a prompt's embeddings; a real one attends among the prompt's own tokens here.)  Returns the slots
        whose prompt found no room: nothing of them was stored."""
        m = self.m
        n_new = [len(prompts.get(b, ())) for b in range(self.B)]
        self.fill.n_new.copy_(torch.tensor(n_new, dtype=torch.int32))
        rows = sum(n_new)
        slots, positions = self._slots(rows)
        tv.paged_plan(None, self.fill, slots, positions, self.status, self.plan, pool=self.pool)
        refused = [b for b, why in enumerate(self.status.tolist()) if why and b in prompts]
        prompts = {b: tokens for b, tokens in prompts.items() if b not in refused}
        tokens = [t for b in range(self.B) for t in prompts.get(b, ())]
        x = m.embed[torch.tensor(tokens, dtype=torch.int64, device="cuda")]
        for layer in range(m.layers):
            self._layer(layer, x, slots[:len(tokens)], positions[:len(tokens)], attend=False)
        self.req.lens.add_(self.fill.n_new * (self.status == 0))
        for b, tokens in prompts.items():
            # the last prompt token is the root of the first tree: its keys come with that
            self.req.lens[b] -= 1
            self.history[b, :len(tokens)] = torch.tensor(tokens, dtype=torch.int32)
            self.said[b] = self.asked[b] = len(tokens)
        return refused

    def finish(self, slot):
        """Ends a request: its pages go back with the next plan."""
        self.req.lens[slot] = 0
        self.req.tree[slot] = -1

    def step(self, trees, draft):
        """One step: trees int32 [B] (bank ids, -1: none), draft int32 [rows] (roots: the last token), the
        trees' nodes one after the other.  A request that finds no room waits: its length stays."""
        m = self.m
        self.req.tree.copy_(trees)
        slots, positions = self._slots(self.rows)
        tv.paged_plan(self.bank, self.req, slots, positions, self.status, self.plan, pool=self.pool, n_q_heads=m.Hq,
                      n_kv_heads=m.H)
        draft = self._drafted_rows(draft)
        x = m.embed[draft.long()]
        for layer in range(m.layers):
            x = self._layer(layer, x, slots, positions, attend=True)
        logits = (x @ m.head).float()
        argmax = torch.zeros(self.rows, dtype=torch.int32, device="cuda")
        tv.logits_process(self.bank, self.req, logits, logits, self.logit_ws, draft=draft, history=self.history,
                          history_len=self.said, prompt_len=self.asked, repetition=self.penalty,
                          presence=self.presence, argmax=argmax)
        accept = tv.paged_accept_q4 if self.q4 else tv.paged_accept
        accept(self.bank, self.req, self.pages, self.results, draft=draft, argmax=argmax, vocab=m.vocab)
        self._note(draft)
        return logits, argmax

    def _drafted_rows(self, draft):
        """The draft tokens in the plan's rows, which leave out the requests that it refused (on the GPU)."""
        drafted = torch.where(self.req.tree < 0, 0, self.nodes[self.req.tree.long()])
        first = drafted.cumsum(0) - drafted
        row = torch.arange(self.rows, dtype=torch.int32, device="cuda")
        b = torch.searchsorted(self.req.row_start[1:], row, right=True).clamp(max=self.B - 1)
        at = first[b] + row - self.req.row_start[b]
        return torch.where(row < self.req.row_start[-1], draft[at.clamp(0, self.rows - 1)], 0)

    def _note(self, draft):
        """Appends the accepted drafts and the bonus token of every request to its history (on the GPU)."""
        n = self.results[:, 0]
        step = torch.arange(64, device="cuda")
        path = self.results[:, 4:].long()
        # token k of the step: the draft of path node k + 1, at the end the bonus token
        nxt = torch.gather(path, 1, (step + 1).clamp(max=63).expand(self.B, 64))
        row = self.req.row_start[:-1, None].long() + nxt
        token = torch.where(step + 1 < n[:, None], draft[row.clamp(max=self.rows - 1)], self.results[:, 1:2])
        at = (self.said[:, None] + step).clamp(max=self.history.shape[1] - 1).long()
        keep = torch.gather(self.history, 1, at)
        self.history.scatter_(1, at, torch.where(step < n[:, None], token, keep))
        self.said.add_(n)


def drafts(server: Server, trees):
    """Draft tokens for the rows of a step: the root is a request's last token, child r of a node the model's
    r-th guess after that node's token without any attention (a real server asks its draft heads)."""
    m = server.m
    guess = (m.embed @ m.head).float().topk(4).indices.int()  # the same for every step: a server keeps it
    out = torch.zeros(server.rows, dtype=torch.int32, device="cuda")
    at = 0
    for b, t in enumerate(trees):
        if t < 0:
            continue
        parent = server.parents[t]
        depth, rank = [0] * len(parent), [0] * len(parent)
        for j in range(1, len(parent)):
            depth[j] = depth[parent[j]] + 1
            rank[j] = sum(1 for i in range(1, j) if parent[i] == parent[j])
        out[at] = server.history[b, server.said[b].long() - 1]
        for level in range(1, max(depth) + 1):
            nodes = [j for j in range(len(parent)) if depth[j] == level]
            up = torch.tensor([at + int(parent[j]) for j in nodes], device="cuda")
            r = torch.tensor([rank[j] for j in nodes], device="cuda")
            out[torch.tensor([at + j for j in nodes], device="cuda")] = guess[out[up].long(), r]
        at += len(parent)
    return out


def main():
    server = Server(Model(), q4="--q4" in sys.argv[1:])
    server.admit({b: list(range(7 * b + 3, 7 * b + 3 + n)) for b, n in enumerate((5, 40, 17, 100))})
    for step in range(6):
        trees = [(b + step) % 3 for b in range(server.B)]
        if step >= 4:
            trees[1] = -1
            if step == 4:
                server.finish(1)
        server.step(torch.tensor(trees, dtype=torch.int32), drafts(server, trees))
        print("step", step, "accepted", server.results[:, 0].tolist(), "lengths", server.req.lens.tolist(), "pages",
              server.pool.held.tolist(), "free", int(server.pool.state[1]), "status", server.status.tolist())
    assert tv.tb_workspace_status(server.ws) == 0


if __name__ == "__main__":
    main()
