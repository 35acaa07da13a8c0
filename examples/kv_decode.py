"""Decoding with a KV cache that does not fit: the operators on KV blocks and the cipher, on the same blocks.

One attention layer of a batch of requests.  Each step appends every request's new key and value to its current block,
attends over the blocks that are on the GPU and adds up the weight that each has gathered; where a request has more blocks
than its budget, the least of them leave: encrypted from the cache straight into pinned host memory, each under the next
IV.  recall() goes the other way: by the 8-bit bounds of all blocks' keys, which stay on the GPU, the best blocks for the
queries at hand are selected, those that are missing are decrypted and verified back into the cache, and the queries attend
over the selection.

    python examples/kv_decode.py [--requests 4] [--steps 200] [--budget 6]
"""
import argparse
import os
import sys

import numpy as np
import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2411_03357_amd as pgcm

FIRST, LAST = 1, 1      # a request's first block, and the one that it writes to, stay


class Decoder:
    """The state of one layer.  Tables, lengths and what lies where are known on the host, as in a serving runtime; the
    device has copies of what its operators read."""

    def __init__(self, requests, budget, most_tokens, heads=8, kv_heads=2, dim=128, block=16, keep=4, half=torch.bfloat16,
                 decay=0.98):
        self.n, self.budget, self.block, self.keep, self.decay = requests, budget, block, keep, decay
        self.heads, self.kv_heads, self.dim, self.half = heads, kv_heads, dim, half
        self.row = -(-most_tokens // block)
        blocks = requests * (budget + keep * kv_heads + 1)
        # a block as the cipher takes it: keys, then values, of its tokens, in one piece
        self.pool = torch.zeros(blocks, 2, block, kv_heads, dim, dtype=half, device="cuda")
        self.cache = pgcm.KVCache(self.pool[:, 0], self.pool[:, 1])
        self.chunk = self.pool[0].numel() * 2
        self.free = list(range(blocks))
        self.tables = np.full((requests, self.row), -1, np.int32)
        self.lens = np.zeros(requests, np.int32)
        self.weights = torch.zeros(requests, self.row, device="cuda")
        # bounds of every block's keys, wherever the block is: entry request * row + place
        self.bounds = torch.zeros(requests * self.row, kv_heads, 2, dim, dtype=torch.int8, device="cuda")
        self.scales = torch.zeros(requests * self.row, kv_heads, device="cuda")
        self.entries = torch.arange(requests * self.row, dtype=torch.int32, device="cuda").view(requests, self.row)
        angle = torch.arange(most_tokens, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2).double() / dim)
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        self.norms = [torch.ones(dim, dtype=half, device="cuda") for _ in "qk"]
        # ciphertext of blocks on the host, their tags and IVs
        self.key = pgcm.expand_key(os.urandom(32))
        self.iv0, self.sent = os.urandom(12), 0
        self.host = torch.empty(requests * self.row, self.chunk, dtype=torch.uint8, pin_memory=True)
        self.tags = torch.zeros(requests * self.row, 16, dtype=torch.uint8, device="cuda")
        self.ivs = {}
        self.moved = {"out": 0, "in": 0}

    def _device(self, a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def step(self, q, k, v):
        """q [requests][heads][dim], k and v [requests][kv_heads][dim]: one new token each -> its attention"""
        place = self.lens // self.block
        for b in range(self.n):
            if self.lens[b] % self.block == 0:
                self.tables[b, place[b]] = self.free.pop()
        at = self.tables[np.arange(self.n), place]
        positions = self._device(self.lens)
        slots = self._device(at.astype(np.int64) * self.block + self.lens % self.block)
        self.lens += 1
        self.q = torch.empty_like(q)
        pgcm.kv_append(self.cache, q, k, v, positions, slots, self.q, q_weight=self.norms[0], k_weight=self.norms[1],
                       rope=self.rope)
        counts = self._device(((self.lens - 1) % self.block + 1).astype(np.int32))
        entries = self._device((np.arange(self.n) * self.row + place).astype(np.int32))
        pgcm.kv_summarize(self.cache, self._device(at), counts, self.bounds, self.scales, entries=entries)
        out = torch.empty_like(q)
        pgcm.kv_attend(self.cache, self.q, self._device(self.tables), self._device(self.lens), out, weights=self.weights,
                       kept=self.weights, decay=self.decay)
        over = (self.tables >= 0).sum(1) - self.budget
        if (over > 0).any():
            self._evict(np.maximum(over, 0).astype(np.int32))
        return out

    def _evict(self, over):
        most = int(over.max())
        victims = torch.empty(self.n, most, dtype=torch.int32, device="cuda")
        pgcm.kv_evict(self.weights, self._device(self.tables), self._device(self.lens), self.block, self._device(over), victims,
                      first=FIRST, last=LAST, blocks=self.pool.shape[0])
        gone = [(b, int(j)) for b, row in enumerate(victims.cpu().numpy()) for j in row if j >= 0]
        blocks = [int(self.tables[b, j]) for b, j in gone]
        self._encrypt([b * self.row + j for b, j in gone], blocks)
        for (b, j), block in zip(gone, blocks):
            self.tables[b, j] = -1
            self.free.append(block)      # what is written to it next follows on the stream

    def _encrypt(self, places, blocks):
        n = len(places)
        for p in places:
            self.ivs[p] = pgcm.seq_iv_bytes(self.iv0, self.sent)
            self.sent += 1
        tags = torch.empty(n, 16, dtype=torch.uint8, device="cuda")
        pgcm.encrypt_batch(self.key, self._ivs(places), None, None, self._addresses(blocks), np.full(n, self.chunk, np.uint64),
                           self._host(places), tags.view(-1))
        self.tags[torch.tensor(places, device="cuda")] = tags
        self.moved["out"] += n

    def _decrypt(self, places, blocks):
        n = len(places)
        ok = torch.empty(n, dtype=torch.uint8, device="cuda")
        tags = self.tags[torch.tensor(places, device="cuda")].contiguous()
        pgcm.decrypt_verify_batch(self.key, self._ivs(places), None, None, self._host(places),
                                  np.full(n, self.chunk, np.uint64), self._addresses(blocks), tags.view(-1), ok)
        if not bool(ok.all()):
            raise RuntimeError("a block did not come back as it left")
        self.moved["in"] += n

    def _ivs(self, places):
        return self._device(np.frombuffer(bytearray().join(self.ivs[p] for p in places), np.uint8))

    def _addresses(self, blocks):
        return np.array([self.pool[i].data_ptr() for i in blocks], np.uint64)

    def _host(self, places):
        return np.array([self.host[p].data_ptr() for p in places], np.uint64)

    def recall(self):
        """attention of the step's queries over the blocks that suit them best, wherever these are -> (out, selected)"""
        selected = torch.empty(self.n, self.kv_heads, self.keep, dtype=torch.int32, device="cuda")
        lens = self._device(self.lens)
        pgcm.kv_select(self.q, self.entries, lens, self.bounds, self.scales, self.block, selected, first=FIRST, last=LAST)
        wanted = selected.cpu().numpy()
        missing = sorted({(b, int(j)) for b in range(self.n) for j in wanted[b].ravel() if j >= 0 and self.tables[b, j] < 0})
        if missing:
            blocks = [self.free.pop() for _ in missing]
            self._decrypt([b * self.row + j for b, j in missing], blocks)
            for (b, j), block in zip(missing, blocks):
                self.tables[b, j] = block
        out = torch.empty_like(self.q)
        pgcm.kv_attend(self.cache, self.q, self._device(self.tables), lens, out, selected=selected)
        return out, wanted


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--budget", type=int, default=6, help="blocks of a request on the GPU")
    args = ap.parse_args()
    d = Decoder(args.requests, args.budget, args.steps)
    for step in range(args.steps):
        q, k, v = [torch.randn(d.n, h, d.dim, device="cuda").to(d.half) for h in (d.heads, d.kv_heads, d.kv_heads)]
        d.step(q, k, v)
        if step % 50 == 49:
            d.recall()
    torch.cuda.synchronize()
    print("%d steps of %d requests: %d blocks of %d bytes encrypted out of the cache, %d decrypted back, all authentic; "
          "%d of %d blocks on the GPU" % (args.steps, d.n, d.moved["out"], d.chunk, d.moved["in"],
                                           int((d.tables >= 0).sum()), int((-(-d.lens // d.block)).sum())))


if __name__ == "__main__":
    main()
