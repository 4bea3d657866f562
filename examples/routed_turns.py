"""Turns of agent sessions, routed to the instances that hold their KV cache and computed there.

Every turn's prompts are hashed, matched against the block index and routed; the instance that
a request goes to takes the pages of the blocks it holds, computes one attention layer of the
tokens that are left and decodes a few more.  The layer's queries, keys and values come from a
random table by token ID, so a prompt's outputs can be checked: the tokens computed after a
hit give what the whole prompt gives on an instance that holds nothing.

    python examples/routed_turns.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_08565_amd import kv, smetric as S  # noqa: E402
from paper_2607_08565_amd.workload import BLOCK, DEFAULT_PARAMS, config0  # noqa: E402

Q_HEADS, KV_HEADS, DIM, DTYPE, IDS, PLACES = 32, 4, 128, torch.bfloat16, 4096, 8192


class Layer:
    """What stands for a model's layer: a row of queries, keys and values per token ID, norm
    weights and the angles of the positions."""

    def __init__(self, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.qkv = draw(IDS, Q_HEADS + 2 * KV_HEADS, DIM).to(DTYPE)
        w = [(1 + 0.1 * draw(DIM)).to(DTYPE) for _ in "qk"]
        f = 1e6 ** (-torch.arange(DIM // 2, dtype=torch.float64, device="cuda") * 2 / DIM)
        a = torch.arange(PLACES, dtype=torch.float64, device="cuda")[:, None] * f
        self.rotary = kv.Rotary(torch.cat([a.cos(), a.sin()], 1).float(), q_weight=w[0], k_weight=w[1])

    def __call__(self, cache: kv.PagedCache, table, q_off, kv_len, tokens, max_new: int):
        """Attention outputs of a ragged batch of new tokens over the cache, which they enter."""
        x = self.qkv[tokens.long() % IDS]
        q, k, v = x[:, :Q_HEADS], x[:, Q_HEADS:Q_HEADS + KV_HEADS], x[:, Q_HEADS + KV_HEADS:]
        plan = kv.Plan(kv_len.numel(), tokens.numel(), Q_HEADS, KV_HEADS, DIM, max_new).make(q_off, kv_len)
        q = kv.append(cache, table, q_off, kv_len, k, v, q=q, rotary=self.rotary)
        return kv.attend(q, cache, table, plan)


class Instance:
    """An instance's cache: pages of one block each, found by their blocks' chained keys."""

    def __init__(self, n_pages: int):
        self.cache = kv.PagedCache.empty(n_pages, KV_HEADS, DIM, BLOCK, DTYPE)
        self.free, self.page_of = list(range(n_pages))[::-1], {}

    def run(self, layer: Layer, prompts, keys, hits, decode: int):
        """Prefills the prompts (token arrays) behind their hits (blocks of theirs that are
        held), then decodes.  Returns each prompt's outputs of the tokens it computed."""
        lens = [len(p) for p in prompts]
        hits = [min(h, (n - 1) // BLOCK) for h, n in zip(hits, lens)]  # at least the last token is computed
        # requests of one batch do not share what neither holds yet
        rows = [[self.page_of[k] for k in ks[:h]] + [self.free.pop() for _ in range(-(-(n + decode) // BLOCK) - h)]
                for ks, h, n in zip(keys, hits, lens)]
        table = torch.full((len(rows), max(map(len, rows))), -1, dtype=torch.int32)
        for r, pages in enumerate(rows):
            table[r, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        table = table.cuda()
        new = [n - h * BLOCK for n, h in zip(lens, hits)]
        tokens = torch.from_numpy(np.concatenate([p[len(p) - n:] for p, n in zip(prompts, new)])).cuda()
        q_off = torch.tensor([0] + new).cumsum(0).cuda()
        kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        out = layer(self.cache, table, q_off, kv_len, tokens, max(new))
        last = out[q_off[1:] - 1]
        for _ in range(decode):  # the next token's ID is read off the last one's output
            ids = last.float().abs().sum((1, 2)).to(torch.int32) % IDS
            kv_len += 1
            last = layer(self.cache, table, torch.arange(len(rows) + 1, device="cuda"), kv_len, ids, 1)
        for ks, pages in zip(keys, rows):
            for k, page in zip(ks, pages):
                self.page_of.setdefault(k, page)
        return [o.clone() for o in out.split(new)], sum(hits)


def main(n_sess: int = 12, n_turns: int = 3, n_inst: int = 3, decode: int = 4) -> float:
    wl = config0(n_sess=n_sess, n_turns=n_turns, n_inst=n_inst)
    layer = Layer()
    pages = n_turns * n_sess * (int(wl.lens[-1].max()) + decode + BLOCK) // BLOCK
    fleet = [Instance(pages) for _ in range(n_inst)]
    index = S.Index(1 << 16, n_inst)
    worst = 0.0
    for t in range(n_turns):
        b = wl.batch(t)
        blk, nb = S.block_offsets(b.tok_off, BLOCK)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
        blk_off = dev(blk)
        block_keys = S.hash_blocks(dev(b.tokens), dev(b.tok_off), blk_off, nb)
        matched = index.match(block_keys, blk_off, nb)
        target, _ = S.route(matched, dev(b.prompt_len), dev(b.hist_len), dev(b.turn), dev(b.q // 20),
                            DEFAULT_PARAMS)  # a lightly loaded fleet: follow-ups stay
        index.insert(block_keys, blk_off, nb, target, dev(b.session.astype(np.int32)), t)
        to, c, keys = target.cpu().numpy(), matched.cpu().numpy(), block_keys.cpu().numpy()
        cached = 0
        for i, inst in enumerate(fleet):
            mine = np.nonzero(to == i)[0]
            if not len(mine):
                continue
            prompts = [b.tokens[b.tok_off[r]:b.tok_off[r + 1]] for r in mine]
            chains = [keys[blk[r]:blk[r + 1]].tolist() for r in mine]
            outs, held = inst.run(layer, prompts, chains, [int(c[r, i]) for r in mine], decode)
            cached += held * BLOCK
            alone, _ = Instance(pages).run(layer, prompts, chains, [0] * len(mine), 0)
            for x, y in zip(outs, alone):
                worst = max(worst, float((x.float() - y[-len(x):].float()).abs().max()))
        print(f"turn {t}: {n_sess} prompts, {b.n_tokens} tokens, {cached} of them held by their instances")
    print(f"largest difference from prompts computed whole: {worst:.3g}")
    return worst


if __name__ == "__main__":
    main()
