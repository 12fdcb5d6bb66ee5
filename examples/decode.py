"""A small decoder that runs both halves of a layer through the library: attention over a paged key-value cache (KVCache) and the sparse FFN over
its neuron cache (Layer).  Random weights; what it shows is the order of the calls.

    python examples/decode.py
    python examples/decode.py --packed         # projections and logits with weights in 4 bits, norms with the residual's addition in one call

    prompts in pieces      reserve -> per layer: append (norms, rotation, keys and values into their pages), attend, FFN
    beams                  fork: sequences that share the pages of a prompt
    decode                 one token per sequence and step
    verification           several drafted tokens of one sequence in a pass, the rejected ones given back (truncate)
    sequences that end     truncate to 0, then compact: the pages in use are the lowest ones again
"""
from __future__ import annotations

import dataclasses
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2312_11514_amd as lif  # noqa: E402
import workloads as wl  # noqa: E402
from workloads.device import GpuLayer  # noqa: E402

FFN_ROWS = 8          # tokens that one FFN step takes


class Decoder:
    """Layers of: x += attention(norm(x)); x += ffn(norm(x)).  Sequences are slots of the key-value cache.  packed: the resident matrices in 4 bits, and the
    rows that they take in 8."""

    def __init__(self, *, layers=2, d_model=512, d_ffn=2048, heads=8, kv_heads=2, vocabulary=1000, page_tokens=16, pages=64, max_seqs=8, max_pages=16,
                 max_tokens=16, dense=False, packed=False, seed=0):
        self.heads, self.kv_heads, self.dim, self.seqs = heads, kv_heads, d_model // heads, max_seqs
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *shape: (torch.randn(*shape, generator=gen) / shape[0] ** 0.5).half().cuda()
        self.embedding = (torch.randn(vocabulary, d_model, generator=gen)).half().cuda()
        self.qkv = [rand(d_model, (heads + 2 * kv_heads) * self.dim) for _ in range(layers)]
        self.out = [rand(d_model, d_model) for _ in range(layers)]
        self.packed = packed
        if packed:
            self.qkv, self.out = ([_packed(w.T.contiguous()) for w in ws] for ws in (self.qkv, self.out))
            self.head = _packed(self.embedding)
        self.norm = [tuple(torch.ones(self.dim, device="cuda") if i % 2 == 0 else None for i in range(4)) for _ in range(layers)]
        self.kv = lif.KVCache(layers=layers, heads=heads, kv_heads=kv_heads, head_dim=self.dim, page_tokens=page_tokens, pages=pages, max_seqs=max_seqs,
                              max_pages=max_pages, max_tokens=max_tokens, norm=lif.NORM_RMS, rotary_dim=self.dim,
                              frequencies=lif.rope_frequencies(self.dim))
        w = wl.scaled(wl.WORKLOADS["C1"], name="decode", d_model=d_model, d_ffn=d_ffn, rank=64, p_active=0.1, dtype="f16", batch=FFN_ROWS,
                      capacity_rows=d_ffn)
        self.ffn = []
        for l in range(layers):
            data = wl.make_layer(w, l)
            if dense:                                      # every neuron predicted active: an FFN that does not depend on the past
                data = dataclasses.replace(data, theta=-1e30)
            self.ffn.append(GpuLayer(w, data))

    def step(self, tokens):
        """tokens: per slot a list of new token numbers (empty: the sequence rests).  Returns logits of the last token of every slot that has
        new ones, {slot: [vocabulary]}, and logits of all new tokens, {slot: [n, vocabulary]}."""
        slots = [s for s, t in enumerate(tokens) if t]
        longest = max(len(tokens[s]) for s in slots)
        counts = torch.tensor([len(t) for t in tokens], dtype=torch.int32).cuda()
        rows = torch.tensor([t + [0] * (longest - len(t)) for t in (tokens[s] for s in slots)]).cuda()
        valid = torch.tensor([i * longest + j for i, s in enumerate(slots) for j in range(len(tokens[s]))]).cuda()
        of_slot = torch.tensor(slots, dtype=torch.int32).cuda()
        self.kv.reserve(counts)
        x = self.embedding[rows]                                                  # [slots, longest, d_model]
        if self.packed:
            logits = self._step_packed(x, valid, of_slot)
            return {s: logits[i, :len(tokens[s])] for i, s in enumerate(slots)}
        h, k = self.heads, self.kv_heads
        for l in range(len(self.ffn)):
            qkv = _normed(x) @ self.qkv[l]
            q, key, value = (t.unflatten(-1, (-1, self.dim)) for t in qkv.split((h * self.dim, k * self.dim, k * self.dim), -1))
            turned = torch.empty(q.shape, dtype=q.dtype, device="cuda")
            mixed = torch.empty_like(turned)
            self.kv.append(l, q, key, value, turned, norm=self.norm[l], slots=of_slot)
            self.kv.attend(l, turned, mixed, slots=of_slot)
            x = x + mixed.flatten(-2) @ self.out[l]
            flat = _normed(x).flatten(0, 1)[valid]
            y = torch.empty_like(flat)
            for at in range(0, len(flat), FFN_ROWS):
                part = flat[at:at + FFN_ROWS]
                self.ffn[l].layer.step(part, y[at:at + FFN_ROWS], len(part))
            x = x.flatten(0, 1).index_add(0, valid, y).unflatten(0, (len(slots), longest))
        logits = (_normed(x) @ self.embedding.T.contiguous()).float()
        return {s: logits[i, :len(tokens[s])] for i, s in enumerate(slots)}

    def _step_packed(self, x, valid, of_slot):
        """The same layers: every norm adds what the half before it has left, and the rows that a matrix in 4 bits takes are rounded to 8 bits."""
        d, shape = x.shape[-1], x.shape[:-1]
        make = lambda *more, dtype=torch.float16: torch.empty(*shape, *more, dtype=dtype, device="cuda")
        codes, scales, normed, y = make(d, dtype=torch.int8), make(1, dtype=torch.float32), make(d), None
        qkv = make((self.heads + 2 * self.kv_heads) * self.dim)
        q, key, value = (t.unflatten(-1, (-1, self.dim)) for t in
                         qkv.split((self.heads * self.dim, self.kv_heads * self.dim, self.kv_heads * self.dim), -1))
        turned, mixed = make(self.heads, self.dim), make(self.heads, self.dim)
        for l in range(len(self.ffn)):
            if y is None:
                lif.add_norm(x, codes, scales=scales)
            else:
                lif.add_norm(y, codes, residual=x, total=x, scales=scales)
            self.qkv[l].multiply(codes, qkv, scales=scales)
            self.kv.append(l, q, key, value, turned, norm=self.norm[l], slots=of_slot)
            self.kv.attend(l, turned, mixed, slots=of_slot)
            lif.add_norm(mixed.flatten(-2), codes, norm=lif.NORM_NONE, scales=scales)
            y = make(d)
            self.out[l].multiply(codes, y, scales=scales)
            lif.add_norm(y, normed, residual=x, total=x)
            flat = normed.flatten(0, 1)[valid]
            ffn = torch.empty_like(flat)
            for at in range(0, len(flat), FFN_ROWS):
                self.ffn[l].layer.step(flat[at:at + FFN_ROWS], ffn[at:at + FFN_ROWS], min(FFN_ROWS, len(flat) - at))
            y = torch.zeros_like(normed)
            y.view(-1, d)[valid] = ffn
        lif.add_norm(y, normed, residual=x, total=x)
        logits = make(self.head.n_out)
        self.head.multiply(normed, logits)
        return logits.float()

    def truncate(self, lengths):
        """{slot: tokens to keep}"""
        self.kv.truncate(torch.tensor([lengths.get(s, -1) for s in range(self.seqs)], dtype=torch.int32).cuda())

    def fork(self, source, slots):
        make = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
        self.kv.fork(make([source] * len(slots)), make(slots))


def _packed(weight):
    matrix = lif.PackedLinear(*weight.shape, group=64, zeros=True)
    matrix.quantize(weight)
    return matrix


def _normed(x):
    f = x.float()
    return (f * torch.rsqrt((f * f).mean(-1, keepdim=True) + 1e-5)).half()


def main(steps=16, drafted=4, **options):
    model = Decoder(**options)
    gen = torch.Generator().manual_seed(1)
    seqs = {s: torch.randint(1000, (n,), generator=gen).tolist() for s, n in ((0, 37), (1, 18), (2, 5))}

    def advance(new):
        return model.step([new.get(s, []) for s in range(model.seqs)])

    last = {}
    for at in range(0, 48, 16):                            # prompts in pieces of up to 16 tokens
        pieces = {s: t[at:at + 16] for s, t in seqs.items() if t[at:at + 16]}
        if pieces:
            last.update({s: l[-1] for s, l in advance(pieces).items()})
    model.fork(0, [3, 4])                                  # three beams of the first prompt, each with another first token
    best = last[0].topk(3).indices.tolist()
    for s, token in zip((0, 3, 4), best):
        seqs[s] = list(seqs[0][:37]) + [token]
    for s in (1, 2):
        seqs[s].append(int(last[s].argmax()))
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(steps):                                 # decode: one token per sequence
        for s, logits in advance({s: t[-1:] for s, t in seqs.items()}).items():
            seqs[s].append(int(logits[-1].argmax()))
    torch.cuda.synchronize()
    us = (time.perf_counter() - start) / steps * 1e6
    draft = torch.randint(1000, (drafted,), generator=gen).tolist()           # verification of one sequence's drafted tokens
    got = advance({2: seqs[2][-1:] + draft})[2].argmax(-1).tolist()
    accepted = next((i for i, (a, b) in enumerate(zip(draft, got)) if a != b), drafted)
    model.truncate({2: len(seqs[2]) + accepted})
    seqs[2] += draft[:accepted] + [got[accepted]]
    before = model.kv.state()["used_pages"]
    model.truncate({1: 0, 3: 0})                           # two sequences end
    model.kv.compact()
    state = model.kv.state()
    for s in (1, 3):
        del seqs[s]
    final = {s: l[-1] for s, l in advance({s: t[-1:] for s, t in seqs.items()}).items()}
    assert model.kv.state()["error"] == 0 and all(f.layer.state()["error"] == 0 for f in model.ffn)
    return {"model": model, "sequences": seqs, "logits": final, "us_per_step": us, "pages_before": before, "pages": state["used_pages"],
            "moved": state["moved_pages"], "accepted": accepted}


if __name__ == "__main__":
    result = main(packed="--packed" in sys.argv[1:])
    print("decode step of 5 sequences, 2 layers: %.0f us (eager)" % result["us_per_step"])
    print("%d of 4 drafted tokens accepted; pages in use %d -> %d after two sequences ended, %d moved" %
          (result["accepted"], result["pages_before"], result["pages"], result["moved"]))
    for slot, tokens in sorted(result["sequences"].items()):
        print("sequence %d: %d tokens, last %s" % (slot, len(tokens), tokens[-5:]))
