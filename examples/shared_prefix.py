"""Block-wise diffusion decoding of several requests of unequal lengths under one shared prefix.

A small randomly initialised model (LLaDA's architecture with norms of queries and keys) runs over the paged
cache of the serving operators: the prefix is computed and stored once, each request's prompt and blocks live
in its own pages, and every step plans pages and slots on the GPU, normalises, rotates and stores queries, keys
and values, attends, and takes its decisions from penalised, biased and grammar-masked logits.  Projections are
the library's too.

    python examples/shared_prefix.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_13740_gb300 import COMMITTED, MASKED, Sched, dllm_op_commit, dllm_op_gemm  # noqa: E402
from paper_2606_13740_gb300.serve import Serve, ServeConfig, dllm_serve_logits  # noqa: E402

D, H, HKV, HD, FFN, VOCAB, LAYERS = 256, 4, 2, 64, 512, 1024, 2
MASK_ID, BLOCK, EPS = VOCAB - 1, 16, 1e-5


class Model:
    """Random bf16 weights; a layer's cache is two pools of pages, numbered alike in all layers."""

    def __init__(self, n_pages, page, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return (torch.randn(*shape, device="cuda", generator=g) * 0.08).to(torch.bfloat16)

        self.embed, self.head = w(VOCAB, D) * 12, w(VOCAB, D)
        self.layers = [dict(qkv=w((H + 2 * HKV) * HD, D), o=w(D, H * HD), up=w(2 * FFN, D), down=w(D, FFN),
                            kc=torch.zeros(n_pages, HKV, page, HD, device="cuda", dtype=torch.bfloat16),
                            vc=torch.zeros(n_pages, HKV, page, HD, device="cuda", dtype=torch.bfloat16),
                            gains=[1 + 0.1 * torch.randn(HD, device="cuda", generator=g) for _ in range(2)])
                       for _ in range(LAYERS)]
        self.theta = 10000.0 ** (-torch.arange(0, HD, 2, device="cuda", dtype=torch.float32) / HD)

    def forward(self, serve, ids, prefix_pages):
        """Hidden states of the plan's rows (ids [rows]); their keys and values go to the planned slots."""
        def norm(x):
            return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)).to(torch.bfloat16)

        rows = ids.numel()
        x = self.embed[ids.long()].float()
        for p in self.layers:
            qkv = dllm_op_gemm(p["qkv"], norm(x), (H + 2 * HKV) * HD, rows, D)
            q, k, v = qkv.split([H * HD, HKV * HD, HKV * HD], 1)
            q = serve.dllm_serve_qk_norm_rope(q, k, v, self.theta, p["kc"], p["vc"], *p["gains"], eps=EPS)
            a = serve.dllm_serve_attention(q, p["kc"], p["vc"], prefix_pages)
            x = x + dllm_op_gemm(p["o"], a, D, rows, H * HD)
            gate, up = dllm_op_gemm(p["up"], norm(x), 2 * FFN, rows, D).chunk(2, 1)
            x = x + dllm_op_gemm(p["down"], (torch.nn.functional.silu(gate) * up).to(torch.bfloat16), D, rows, FFN)
        return norm(x)

    def logits(self, hidden):
        return dllm_op_gemm(self.head, hidden, VOCAB, hidden.shape[0], D)


class Batch:
    """Requests under a shared prefix.  The prefix is a request of its own, in the last row of the tables, which
    only holds its pages once it is computed."""

    def __init__(self, prefix, prompts, gen_len, page=16, seed=0):
        self.B, self.P = len(prompts), len(prefix)
        n_own = [-(-(len(p) + gen_len) // page) for p in prompts]
        n_pages = sum(n_own) + -(-self.P // page)
        self.serve = Serve(ServeConfig(max_batch=self.B + 1, max_rows=max(self.P, sum(len(p) for p in prompts), self.B * BLOCK),
                                       page=page, n_pages=n_pages, max_pages=max(n_own + [-(-self.P // page)]), n_heads=H,
                                       n_kv_heads=HKV, head_dim=HD))
        self.model = Model(n_pages, page, seed)
        self.tokens = [list(p) for p in prompts]  # of each request, without the prefix
        self.pages = None
        self.len = np.zeros(self.B, np.int32)  # own positions whose keys and values are final
        if self.P:
            self._run([0] * self.B, [0] * self.B, [prefix])
            self.pages = self.serve.table[self.B, :-(-self.P // page)].clone()
        self._run(self.len, [len(p) for p in prompts], prompts)
        self.len[:] = [len(p) for p in prompts]

    def _run(self, length, q_len, ids):
        """A forward pass over new tokens (ids, request by request) behind `length` own positions."""
        first = self.pages is None and self.P  # the prefix itself
        i32 = dict(dtype=torch.int32, device="cuda")
        L = torch.tensor(list(length) + [0 if first else self.P], **i32)
        Q = torch.tensor(list(q_len) + [self.P if first else 0], **i32)
        flat = torch.tensor([t for r in ids for t in r], **i32)
        self.serve.dllm_serve_plan(L, Q, flat.numel(), prefix_len=0 if first else self.P)
        return self.model.forward(self.serve, flat, self.pages)

    def block_logits(self):
        """Logits of the next block, all of it masked."""
        hidden = self._run(self.len, [BLOCK] * self.B, [[MASK_ID] * BLOCK] * self.B)
        return self.model.logits(hidden)

    def decode_block(self, steps=4, rep=1.2, freq=0.1, pres=0.1, grammar=None, bias=None):
        """The next block of every request, committed over `steps` passes; bias: {id: value}, grammar: ids allowed."""
        B, T = self.B, BLOCK
        i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
        tok = np.full((B, T), MASK_ID, np.int32)
        state = np.full((B, T), MASKED, np.uint8)
        words = torch.full((1, (VOCAB + 31) // 32), -1, **i32)
        if grammar is not None:
            bits = np.zeros(32 * words.shape[1], np.uint8)
            bits[list(grammar)] = 1
            words[0] = torch.from_numpy(np.packbits(bits, bitorder="little").view(np.int32)).cuda()
        for step in range(steps):
            z = self.model.logits(self._run(self.len, [T] * B, tok.tolist()))
            seen = [t + [v for v in row if v != MASK_ID] for t, row in zip(self.tokens, tok.tolist())]
            longest = max(len(s) for s in seen)
            x0, conf, tokconf = dllm_serve_logits(
                z, MASK_ID, req=torch.arange(B, **i32).repeat_interleave(T),
                hist=torch.tensor([s + [-1] * (longest - len(s)) for s in seen], **i32),
                hist_len=torch.tensor([len(s) for s in seen], **i32), rep=torch.full((B,), rep, **f32),
                freq=torch.full((B,), freq, **f32), pres=torch.full((B,), pres, **f32),
                bias_ids=None if not bias else torch.tensor([list(bias)] * B, **i32),
                bias=None if not bias else torch.tensor([list(bias.values())] * B, **f32),
                grammar=words, grammar_row=torch.zeros(B * T, **i32),
                cur=torch.tensor(tok.ravel(), **i32), out=z)
            x0, conf, tokconf = (v.cpu().numpy().reshape(B, T) for v in (x0, conf, tokconf))
            for b in range(B):
                tok[b], state[b], _ = dllm_op_commit(Sched(steps_per_block=steps), MASK_ID, tok[b], state[b], 0, T, 0, T, step,
                                                     x0[b], conf[b], tokconf[b], block_len=T)
        assert (state == COMMITTED).all()
        # the last pass still held masks: keys and values again, from the final ids
        self._run(self.len, [T] * B, tok.tolist())
        self.serve.dllm_serve_check()
        for t, row in zip(self.tokens, tok.tolist()):
            t += row
        self.len += T
        return tok


def main():
    rng = np.random.default_rng(0)
    prefix = rng.integers(0, MASK_ID, 200).tolist()
    prompts = [rng.integers(0, MASK_ID, n).tolist() for n in (5, 37, 1, 64)]
    batch = Batch(prefix, prompts, gen_len=3 * BLOCK)
    for _ in range(3):
        batch.decode_block(grammar=range(0, MASK_ID, 2), bias={10: 1.0, 20: -100.0})
    for n, t in zip((len(p) for p in prompts), batch.tokens):
        print(f"prompt of {n:3d}: {t[n:]}")


if __name__ == "__main__":
    main()
