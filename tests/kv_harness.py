"""Test-side glue of the key-value cache: builds a cache with scattered pages, and reads pages back in their natural order."""
from __future__ import annotations

import numpy as np
import torch

import paper_2312_11514_amd as lif
from workloads.device import require_gpu

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # largest relative error of one rounding


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def build(lengths, fresh, *, kv_heads, head_dim, page, dtype, seed, heads=None, layers=2, layer=1, spare=3, garbage=float("nan"), max_tokens=None,
          slots=None, max_seqs=None, max_pages=0, **more):
    """A cache whose sequences (batch row i in slot slots[i]) hold random keys and values in layer `layer`, pages scattered over the pool,
    and `garbage` everywhere else: in free pages, in other layers, behind the last token of a page.
    Returns the cache and the fp64 keys and values per row, [kv_heads, n, head_dim]."""
    require_gpu()
    rng = np.random.default_rng(seed)
    per = [-(-n // page) for n in lengths]
    slots = list(range(len(lengths))) if slots is None else slots
    max_seqs, max_pages = max_seqs or max(slots) + 1, max(per + [1, max_pages])
    kv = lif.KVCache(layers=layers, heads=heads or kv_heads, kv_heads=kv_heads, head_dim=head_dim, page_tokens=page, pages=sum(per) + spare,
                     max_seqs=max_seqs, max_pages=max_pages, max_tokens=max_tokens or max(list(fresh) + [1]), dtype=dtype, **more)
    order = rng.permutation(sum(per) + spare).tolist()
    table = np.full((max_seqs, max_pages), -1, np.int32)
    n_of, f_of = np.zeros(max_seqs, np.int32), np.zeros(max_seqs, np.int32)
    kv.k.fill_(garbage)
    kv.v.fill_(garbage)
    rows = []
    for slot, n, f, p in zip(slots, lengths, fresh, per):
        pages = [order.pop() for _ in range(p)]
        table[slot, :p], n_of[slot], f_of[slot] = pages, n, f
        keys = torch.from_numpy(rng.standard_normal((kv_heads, n, head_dim), dtype=np.float32)).to(DTYPES[dtype])
        values = torch.from_numpy(rng.standard_normal((kv_heads, n, head_dim), dtype=np.float32)).to(DTYPES[dtype])
        put(kv, layer, pages, keys, values)
        rows.append((keys.double().numpy(), values.double().numpy()))
    kv.table.copy_(torch.from_numpy(table))
    kv.lengths.copy_(torch.from_numpy(n_of))
    kv.fresh.copy_(torch.from_numpy(f_of))
    kv.adopt()
    return kv, rows


def put(kv, layer, pages, keys, values, first=0):
    """Writes keys and values [kv_heads, n, head_dim] as the tokens first .. first + n - 1 of a sequence."""
    page = kv.k.shape[3]
    e = kv.v.shape[5]
    for j, p in enumerate(pages):
        lo, hi = max(j * page, first), min((j + 1) * page, first + keys.shape[1])
        if hi <= lo:
            continue
        kv.k[layer, p, :, lo - j * page:hi - j * page] = keys[:, lo - first:hi - first].to(kv.k.device)
        v = kv.v[layer, p].permute(0, 1, 3, 2).reshape(keys.shape[0], page, -1)
        v[:, lo - j * page:hi - j * page] = values[:, lo - first:hi - first].to(kv.v.device)
        kv.v[layer, p] = v.reshape(keys.shape[0], page // e, e, -1).permute(0, 1, 3, 2)


def get(kv, layer, pages):
    """Keys and values of pages in order, [kv_heads, tokens, head_dim], on the CPU."""
    k = kv.k[layer, pages].cpu()
    v = kv.v[layer, pages].cpu()
    h, d = k.shape[1], k.shape[3]
    return (k.permute(1, 0, 2, 3).reshape(h, -1, d), v.permute(1, 0, 2, 4, 3).reshape(h, -1, d))
