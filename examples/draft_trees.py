"""Greedy decoding from trees of drafts, and beam search on shared pages, with the serving operators.

A small randomly initialised causal model (that of shared_prefix.py) decodes several requests at once.  `Drafted` lets
every request guess a tree of tokens from what it has seen (what followed its last token before, and any tokens),
checks all guesses in one pass, and keeps the path that the model's decisions bear out: one to several tokens a pass.
`Beams` forks a prompt into beams, scored by log probabilities, that share the pages they have in common.

    python examples/draft_trees.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from shared_prefix import EPS, FFN, H, HD, HKV, LAYERS, VOCAB, D, Model  # noqa: E402

from paper_2606_13740_gb300 import dllm_op_gemm  # noqa: E402
from paper_2606_13740_gb300.serve import Serve, ServeConfig, dllm_serve_logits, dllm_serve_logprobs  # noqa: E402

TREE = 12  # tokens of a tree, the one decided on among them


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Causal:
    """Requests of one batch over a paged cache: prompts first, then whatever the subclass does."""

    def __init__(self, prompts, n_pages, max_pages, rows, batch=None, page=16, seed=0):
        self.model = Model(n_pages, page, seed)
        self.serve = Serve(ServeConfig(max_batch=batch or len(prompts), max_rows=max(rows, sum(map(len, prompts))), page=page,
                                       n_pages=n_pages, max_pages=max_pages, n_heads=H, n_kv_heads=HKV, head_dim=HD))
        self.layers = self.serve.layers([p["kc"] for p in self.model.layers], [p["vc"] for p in self.model.layers])
        L, Q = i32([0] * len(prompts)), i32([len(p) for p in prompts])
        self.serve.dllm_serve_plan(L, Q, sum(map(len, prompts)), causal=True)
        z = self.logits(i32([t for p in prompts for t in p]))
        self.len = Q
        self.last = z[torch.cumsum(Q, 0).long() - 1]  # logits behind each prompt

    def logits(self, ids, mask=None):
        """Logits of the plan's rows, attended by bits where there are some."""
        def norm(x):
            return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)).to(torch.bfloat16)

        m, s, rows = self.model, self.serve, ids.numel()
        x = m.embed[ids.long()].float()
        for p in m.layers:
            q, k, v = dllm_op_gemm(p["qkv"], norm(x), (H + 2 * HKV) * HD, rows, D).split([H * HD, HKV * HD, HKV * HD], 1)
            q = s.dllm_serve_qk_norm_rope(q, k, v, m.theta, p["kc"], p["vc"], *p["gains"], eps=EPS)
            if mask is None:
                a = s.dllm_serve_attention(q, p["kc"], p["vc"])
            else:
                a = s.dllm_serve_tree_attention(q, p["kc"], p["vc"], mask)
            x = x + dllm_op_gemm(p["o"], a, D, rows, H * HD)
            gate, up = dllm_op_gemm(p["up"], norm(x), 2 * FFN, rows, D).chunk(2, 1)
            x = x + dllm_op_gemm(p["down"], (torch.nn.functional.silu(gate) * up).to(torch.bfloat16), D, rows, FFN)
        return m.logits(norm(x))


class Drafted(Causal):
    def __init__(self, prompts, gen_len, seed=0):
        need = [-(-(len(p) + gen_len + 2 * TREE) // 16) for p in prompts]
        super().__init__(prompts, sum(need), max(need), TREE * len(prompts), seed=seed)
        self.tokens = [list(p) for p in prompts]
        self.next = dllm_serve_logits(self.last)[0].tolist()  # decided on, not yet in the cache
        self.rng = np.random.default_rng(seed)
        self.seen = []  # (request, token's place, logits of its row): what the decisions were taken from

    def guess(self, b):
        """A tree behind the token decided on: (parents, ids).  Two chains of what followed its last occurrences, else any."""
        past, ids, parent = self.tokens[b] + [self.next[b]], [self.next[b]], [-1]
        places = [i for i in range(len(past) - 1) if past[i] == past[-1]][-2:]
        for at in places:
            node = 0
            for t in past[at + 1:at + 4]:
                parent.append(node)
                ids.append(t)
                node = len(ids) - 1
        while len(ids) < TREE:
            parent.append(int(self.rng.integers(0, len(ids))))
            ids.append(int(self.rng.integers(0, VOCAB)))
        return parent, ids

    def step(self):
        """One pass: every request's tree is checked, its path kept.  Returns the tokens that each request gained."""
        s, B = self.serve, len(self.tokens)
        trees = [self.guess(b) for b in range(B)]
        parent, ids = i32([p for t, _ in trees for p in t]), i32([t for _, u in trees for t in u])
        s.dllm_serve_plan(self.len, i32([TREE] * B), TREE * B)
        mask = s.dllm_serve_tree(parent, TREE)
        z = self.logits(ids, mask)
        x0, _, _ = dllm_serve_logits(z)
        keep, n, nxt = s.dllm_serve_accept(parent, ids, x0, B, TREE)
        s.dllm_serve_compact(self.layers, self.len, keep, n)
        s.dllm_serve_check()
        gained = []
        for b, (path, count) in enumerate(zip(keep.tolist(), n.tolist())):
            gained.append([trees[b][1][j] for j in path[:count]])
            self.seen += [(b, len(self.tokens[b]) + i, z[TREE * b + j]) for i, j in enumerate(path[:count])]
            self.tokens[b] += gained[b]
        self.len, self.next = self.len + n, nxt.tolist()
        return gained


class Beams(Causal):
    def __init__(self, prompt, beams, gen_len, seed=0):
        need = -(-(len(prompt) + gen_len + 1) // 16)
        super().__init__([prompt], need + beams * (1 + -(-gen_len // 16)) + beams, need + 1, beams, batch=beams, seed=seed)
        self.K, self.prompt, self.places = beams, prompt, len(prompt)
        _, _, first, lp, _ = dllm_serve_logprobs(self.last, top=beams)
        self.tokens = first[0, :, None]  # [K][tokens so far]
        self.score = lp[0]
        self._fork(torch.zeros(beams, dtype=torch.int32, device="cuda"))

    def _fork(self, src):
        self.serve.dllm_serve_fork(self.layers, src, torch.full_like(src, self.places))

    def step(self):
        """The beams' last tokens go into the cache, and the K best of their K * K continuations become the beams."""
        K, s = self.K, self.serve
        s.dllm_serve_plan(torch.full((K,), self.places, dtype=torch.int32, device="cuda"), i32([1] * K), K, causal=True)
        self.places += 1
        _, _, ids, lp, _ = dllm_serve_logprobs(self.logits(self.tokens[:, -1].contiguous()), top=K)
        score, at = (self.score[:, None] + lp).flatten().topk(K)
        src = (at // K).to(torch.int32)
        self.tokens = torch.cat([self.tokens[src.long()], ids.flatten()[at][:, None]], 1)
        self.score = score
        self._fork(src)
        s.dllm_serve_check()


def main():
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, VOCAB, n).tolist() for n in (5, 37, 1, 64)]
    d = Drafted(prompts, 40)
    for _ in range(12):
        d.step()
    for n, t in zip(map(len, prompts), d.tokens):
        print(f"prompt of {n:3d}: {len(t) - n} tokens in 12 passes: {t[n:]}")
    b = Beams(prompts[1], 4, 12)
    for _ in range(11):
        b.step()
    for score, t in zip(b.score.tolist(), b.tokens.tolist()):
        print(f"beam {score:8.3f}: {t}")
    print(f"{b.serve.ring_pos[1].item()} of {b.serve.cfg.n_pages} pages free, {LAYERS} layers")


if __name__ == "__main__":
    main()
