"""A long conversation in a small cache: one attention layer whose keys and
values live in a pool of slots, with an index of its keys beside it.

  prompt   read in chunks: each chunk's keys and values are appended to their
           slots, its tokens attend to everything cached, and the attention
           that every cached token draws is summed up
  index    a token that leaves the recent window goes into a GRAND_MIPS index
           of its key/value head; slots are the index's ids
  evict    beyond a budget the tokens that drew the least attention leave the
           cache and the indexes, and their slots are used again
  answer   a new token attends to the recent window, and to the slots that its
           heads' searches return; the two parts are joined

Run: python examples/retrieval_cache.py   (needs an MI355X)
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2608_21163_amd import Cache, GrandIndex
from workloads import IndexConfig

INVALID = -1


class RetrievalLayer:
    """The cache of one sequence and one layer, a slot a page."""

    def __init__(self, q_heads=8, kv_heads=2, dim=64, slots=4096, budget=2048, window=128, sinks=4, k=64, beam=128, max_norm=24.0):
        self.hq, self.hk, self.dim, self.k, self.beam = q_heads, kv_heads, dim, k, beam
        self.budget, self.window, self.sinks = budget, window, sinks
        stream = torch.cuda.current_stream().cuda_stream
        self.cache = Cache("bf16", q_heads, kv_heads, dim, page_size=1, stream=stream)
        self.k_pages = torch.zeros(slots, 1, kv_heads, dim, dtype=torch.bfloat16, device="cuda")
        self.v_pages = torch.zeros_like(self.k_pages)
        config = IndexConfig("vamana", "f32", "mips", dim, slots, 32, 64, mips_norm=max_norm)
        self.index = [GrandIndex.from_config(config, max_batch=1024, stream=stream) for _ in range(kv_heads)]
        self.free = list(range(slots - 1, -1, -1))
        self.table = torch.full((1, slots), INVALID, dtype=torch.int32, device="cuda")
        self.weights = torch.zeros(1, kv_heads, slots, device="cuda")
        self.length = 0          # tokens cached
        self.indexed = 0         # tokens, from the front, that the indexes hold

    def _grow(self, k, v):
        """Slots and places for new tokens; returns the call's sequences."""
        n = k.shape[0]
        slots = torch.tensor([self.free.pop() for _ in range(n)], dtype=torch.int32)
        self.table[0, self.length:self.length + n] = slots.cuda()
        self.length += n
        lens = torch.tensor([self.length], dtype=torch.int32, device="cuda")
        start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        s = self.cache.sequences(self.table, lens, start, max_q=n, max_k=self.length)
        self.cache.append(s, k, v, self.k_pages, self.v_pages)
        return s

    def _index_old(self):
        """Tokens that left the window go into the indexes."""
        last = max(self.sinks, self.length - self.window)
        first, self.indexed = max(self.sinks, self.indexed), max(self.indexed, last)
        if first >= last:
            return
        ids = self.table[0, first:last].contiguous()
        for h, index in enumerate(self.index):
            index.insert(ids, self.k_pages[ids.long(), 0, h].float())

    def _evict(self):
        """Back to the budget: what goes leaves the indexes too."""
        if self.length <= self.budget:
            return
        lens = torch.tensor([self.length], dtype=torch.int32, device="cuda")
        budget = torch.tensor([self.budget], dtype=torch.int32, device="cuda")
        s = self.cache.sequences(self.table, lens, max_k=self.length)
        self.table, self.weights, _, freed, _ = self.cache.evict(s, self.weights, budget, sinks=self.sinks, recent=self.window)
        gone = freed[0, :self.length - self.budget].contiguous()
        for index in self.index:
            index.delete(gone)
        self.free += gone.tolist()
        self.indexed -= gone.numel()
        self.length = self.budget

    def read(self, q, k, v):
        """A chunk of the prompt: attention over everything cached."""
        s = self._grow(k, v)
        out, lse, self.weights = self.cache.attend(s, q, self.k_pages, self.v_pages, weights=self.weights)
        self._index_old()
        self._evict()
        return out, lse

    def answer(self, q, k, v):
        """One new token: the window, the sinks and what the searches return.
        Returns the joined result, and attention over the whole cache beside
        it for comparison."""
        s = self._grow(k, v)
        self._index_old()        # the new token has pushed one out of the window
        near = self.cache.attend(s, q, self.k_pages, self.v_pages, window=self.window)
        ids = torch.full((1, self.hq, self.k + self.sinks), INVALID, dtype=torch.int32, device="cuda")
        group = self.hq // self.hk
        for h, index in enumerate(self.index):
            found = torch.empty(group, self.k, dtype=torch.int32, device="cuda")
            dists = torch.empty(group, self.k, device="cuda")
            index.search(q[0, h * group:(h + 1) * group].float().contiguous(), self.k, self.beam, found, dists)
            ids[0, h * group:(h + 1) * group, :self.k] = found
        out_of_window = min(self.sinks, max(0, self.length - self.window))
        ids[0, :, self.k:self.k + out_of_window] = self.table[0, :out_of_window]
        got = self.cache.attend_ids(q, self.k_pages, self.v_pages, ids, prior=near)
        whole = self.cache.attend(s, q, self.k_pages, self.v_pages)
        self._evict()
        self.cache.check()
        return got, whole

    def close(self):
        self.cache.close()
        for index in self.index:
            index.close()


def conversation(tokens, q_heads, kv_heads, dim, topics=40, seed=0):
    """Queries, keys and values whose attention is peaked: a token's query
    points at the keys of its topic."""
    r = np.random.default_rng(seed)
    centre = r.standard_normal((topics, kv_heads, dim)) * 1.2
    topic = r.integers(0, topics, tokens)
    k = centre[topic] + 0.6 * r.standard_normal((tokens, kv_heads, dim))
    q = np.repeat(centre[topic], q_heads // kv_heads, axis=1) * 1.5 + 0.5 * r.standard_normal((tokens, q_heads, dim))
    v = r.standard_normal((tokens, kv_heads, dim))
    return [torch.from_numpy(x).bfloat16().cuda() for x in (q, k, v)]


def main(prompt=5000, chunk=500, answers=40, seed=0):
    layer = RetrievalLayer()
    q, k, v = conversation(prompt + answers, layer.hq, layer.hk, layer.dim, seed=seed)
    for i in range(0, prompt, chunk):
        layer.read(q[i:i + chunk], k[i:i + chunk], v[i:i + chunk])
    report = []
    for i in range(prompt, prompt + answers):
        (out, lse), (whole, z) = layer.answer(q[i:i + 1], k[i:i + 1], v[i:i + 1])
        report.append(dict(caught=torch.exp(lse - z).cpu().numpy(), error=(out.float() - whole.float()).abs().amax(-1).cpu().numpy(),
                           largest=float(layer.v_pages.float().abs().max())))
    live = [set(np.flatnonzero(index.export()["active"]).tolist()) for index in layer.index]
    table = layer.table[0, :layer.length].tolist()
    used = dict(length=layer.length, slots=len(set(table)), free=len(layer.free),
                indexed=all(s == set(table[layer.sinks:layer.indexed]) for s in live))
    layer.close()
    return report, used


if __name__ == "__main__":
    report, used = main()
    caught = np.concatenate([r["caught"].ravel() for r in report])
    print(f"{used['length']} tokens cached, {used['free']} slots free; the window and the retrieved slots hold "
          f"{caught.mean():.4f} of the attention on average, {caught.min():.4f} at least")
    print(f"largest difference from attention over the whole cache: {max(r['error'].max() for r in report):.4f}")
