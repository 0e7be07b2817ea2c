"""One layer of a serving loop around the coder: a context stored as records is decoded into the pages of a live cache, new tokens
are written into those pages and attend to them, and what leaves the window goes back to the coder.

    stored records -> kvtc_decode -> kvtc_rope -> kvtc_cache_write          the context, restored
    every token:      kvtc_rope, kvtc_cache_write, kvtc_attend              its keys and values, and what it sees
    every STEP tokens: kvtc_cache_read -> kvtc_rope (inverse) -> kvtc_encode   the oldest tokens of the window, stored behind the context

    python examples/paged_decode.py [--context 8192] [--tokens 64] [--sequences 4] [--format fp8]

Inputs are synthetic: tensors on the committed plans' bases.  Prints the time of a token's three calls and of the rest, and checks the last token's attention
against elementary torch operations on what the cache holds.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2511_01815_amd as kv  # noqa: E402
from paper_2511_01815_amd import bundles  # noqa: E402

HEADS, QUERIES, D = 8, 32, 128
WIDE = HEADS * D
PAGE, WINDOW, STEP = 64, 128, 16
BASE = 500000.0
FORMATS = {"bf16": kv.KVTC_CACHE_BF16, "fp8": kv.KVTC_CACHE_FP8, "int4": kv.KVTC_CACHE_INT4}
DEV = "cuda:0"


class Side:
    """Keys or values: the plan, its basis for drawing tensors, the pool of pages and the stored records of every sequence."""

    def __init__(self, bundle, fmt, n_pages, sequences, most_tokens, gen):
        a = bundles.load_plan_arrays(bundle)
        self.plan = kv.Plan(a["mu32"].shape[0], a["v_bits"].shape[1], a["mu32"], a["v_bits"], list(zip(a["group_n"], a["group_bits"])))
        self.mu = torch.from_numpy(a["mu32"]).to(DEV)
        self.basis = torch.from_numpy((a["v_bits"].astype(np.uint32) << 16).view(np.float32)).to(DEV)
        self.size = torch.arange(1, self.basis.shape[1] + 1, device=DEV) ** -0.5
        self.gen = gen
        row, scale = kv.kvtc_cache_row_bytes(fmt, D), kv.kvtc_cache_scale_bytes(fmt, D)
        self.rows = torch.zeros((n_pages, HEADS, PAGE, row), dtype=torch.uint8, device=DEV)
        self.scales = torch.zeros((n_pages, HEADS, PAGE, max(1, scale)), dtype=torch.uint8, device=DEV) if scale else None
        self.records = torch.zeros((sequences, most_tokens * self.plan.record_bytes), dtype=torch.uint8, device=DEV)

    def draw(self, n):
        """n tokens before any rotation."""
        z = torch.randn((n, self.basis.shape[1]), generator=self.gen, device=DEV) * self.size
        return (z @ self.basis.T * 8 + self.mu).to(torch.bfloat16)

    def store(self, b, at, x):
        """Tokens at .. at + len(x) of sequence b, coded."""
        r = self.plan.record_bytes
        kv.kvtc_encode(self.plan.handle, x, kv.KVTC_BF16, len(x), WIDE, self.records[b, at * r:], len(x) * r)

    def restore(self, b, n):
        x = torch.empty((n, WIDE), dtype=torch.bfloat16, device=DEV)
        kv.kvtc_decode(self.plan.handle, self.records[b], n * self.plan.record_bytes, n, x, kv.KVTC_BF16, WIDE)
        return x


def rotate(keys, positions, inverse=False):
    kv.kvtc_rope(keys, kv.KVTC_BF16, keys.shape[0], HEADS, D, WIDE, D, positions, 0, BASE, kv.ROPE_HALF, inverse)


class Session:
    def __init__(self, context, tokens, sequences, fmt, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.fmt, self.context, self.most = FORMATS[fmt], context, context + tokens
        each = -(-self.most // PAGE)
        n_pages = sequences * each
        self.pages = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32).view(sequences, each)
        # (stored starts lie on 16 bytes; STEP records of these plans do)
        self.k, self.v = [Side(f"c2_{s}_cr16", self.fmt, n_pages, sequences, self.most, gen) for s in "KV"]
        s = self.k.rows.stride()
        self.cache = kv.cache(self.fmt, n_pages, PAGE, HEADS, D, self.k.rows, self.v.rows, s[0], s[1], s[2], self.k.scales, self.v.scales)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=DEV)
        self.stored = 0
        self.work = torch.zeros(kv.kvtc_attend_work_bytes(self.cache, sequences, QUERIES, self.most), dtype=torch.uint8, device=DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.gen, self.sequences = gen, sequences
        for b in range(sequences):                               # what an earlier session stored
            for side in (self.k, self.v):
                side.store(b, 0, side.draw(context))

    def slots(self, b, first, n):
        t = torch.arange(first, first + n, device=DEV)
        return self.pages[b].long()[t // PAGE] * PAGE + t % PAGE

    def restore(self):
        """The stored context into pages; its last WINDOW tokens are the window again."""
        for b in range(self.sequences):
            k, v = self.k.restore(b, self.context), self.v.restore(b, self.context)
            rotate(k, torch.arange(self.context, dtype=torch.int32, device=DEV))
            kv.kvtc_cache_write(self.cache, k, v, kv.KVTC_BF16, self.context, WIDE, D, self.slots(b, 0, self.context), self.status)
        self.lengths.fill_(self.context)
        self.stored = max(0, (self.context - WINDOW) // STEP * STEP)

    def token(self, k, v, q):
        """One new token of every sequence: [sequences, WIDE] keys (not yet rotated) and values, [sequences, QUERIES, D] queries -> what they see."""
        rotate(k, self.lengths)
        place = torch.gather(self.pages, 1, (self.lengths // PAGE).long()[:, None])[:, 0].long() * PAGE + self.lengths % PAGE
        kv.kvtc_cache_write(self.cache, k, v, kv.KVTC_BF16, self.sequences, WIDE, D, place, self.status)
        self.lengths += 1
        out = torch.empty_like(q)
        kv.kvtc_attend(self.cache, q, kv.KVTC_BF16, self.sequences, QUERIES, QUERIES * D, D, self.pages, self.pages.shape[1], self.lengths, self.most, D ** -0.5, 0, 0, out, None,
                       self.work, self.work.numel(), self.status)
        return out

    def leave_window(self, length):
        """STEP tokens that no longer belong to the window of `length` tokens' sequences: out of the cache, rotation undone, stored behind those before."""
        if length - self.stored < WINDOW + STEP:
            return False
        at = torch.arange(self.stored, self.stored + STEP, dtype=torch.int32, device=DEV)
        for b in range(self.sequences):
            k, v = [torch.empty((STEP, WIDE), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            kv.kvtc_cache_read(self.cache, self.slots(b, self.stored, STEP), STEP, k, v, kv.KVTC_BF16, WIDE, D, self.status)
            rotate(k, at, inverse=True)
            self.k.store(b, self.stored, k)
            self.v.store(b, self.stored, v)
        self.stored += STEP
        return True

    def seen_plainly(self, q, length):
        """What token() gives, of sequence 0, by elementary operations on the cache's own values."""
        k, v = [torch.empty((length, HEADS, D), device=DEV) for _ in range(2)]
        kv.kvtc_cache_read(self.cache, self.slots(0, 0, length), length, k, v, kv.KVTC_F32, WIDE, D, self.status)
        q = q[0].float().view(HEADS, QUERIES // HEADS, D)
        p = torch.softmax(torch.matmul(q, k.permute(1, 2, 0)) * D ** -0.5, -1)
        return torch.matmul(p, v.permute(1, 0, 2)).reshape(QUERIES, D)


def run(context=8192, tokens=64, sequences=4, fmt="fp8", seed=0):
    s = Session(context, tokens, sequences, fmt, seed)
    torch.cuda.synchronize()
    t = time.perf_counter()
    s.restore()
    torch.cuda.synchronize()
    restored, in_tokens, moved = time.perf_counter() - t, 0.0, 0
    for i in range(tokens):
        k, v, q = s.k.draw(sequences), s.v.draw(sequences), torch.randn((sequences, QUERIES, D), generator=s.gen, device=DEV).to(torch.bfloat16)
        torch.cuda.synchronize()
        t = time.perf_counter()
        out = s.token(k, v, q)
        torch.cuda.synchronize()
        in_tokens += time.perf_counter() - t
        moved += s.leave_window(context + i + 1)
    want = s.seen_plainly(q, context + tokens)
    off = float((out[0].float() - want).norm() / want.norm())
    assert int(s.status.item()) == 0, "a token or a page had no place"
    return {"restore_ms": restored * 1e3, "token_us": in_tokens / tokens * 1e6, "steps_stored": moved, "off": off, "session": s, "out": out}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--context", type=int, default=8192)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--format", choices=sorted(FORMATS), default="fp8")
    a = ap.parse_args()
    for again in range(2):                                       # (the first run pays for loading the kernels)
        r = run(a.context, a.tokens, a.sequences, a.format)
    print(f"{a.sequences} sequences of {a.context} tokens, pages in {a.format}: restored in {r['restore_ms']:.2f} ms; "
          f"{r['token_us']:.0f} us a token of all of them (waited for each time); {r['steps_stored']} x {STEP} tokens stored; "
          f"last token off by {r['off']:.1e} of what the cache's values give")


if __name__ == "__main__":
    main()
