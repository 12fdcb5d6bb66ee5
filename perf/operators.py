"""The attention half of a decode step over a paged key-value cache: what its speed is measured on.

A case is one pass through one of three operators of paper_2312_11514_amd.KVCache:

  op "append"  KVCache.append: norms of queries and keys per head, rotary positions, keys and values written to their pages
  op "attend"  KVCache.attend: attention of the newest tokens of every sequence over the pages of its cache
  op "pages"   the page calls.  kind "verify": pages reserved for the tokens of a speculative pass, all of them given back;
               "fork": every sequence gets `tokens` others that share its full pages and have a copy of its partial last one, after
               the former ones were freed; "burst": all sequences anew, every second one ends, the pages of the others move together

Head layouts are those of the layers this library is measured on (32 heads of 128 for OPT-6.7B and Llama-2-7B, 71 heads of 64 on one
key head for Falcon-7B, 32 heads of 80 with 32 rotated dimensions for Phi-2, 64 heads of 64 with normalised queries and keys for
Persimmon-8B) and, generic, 32 heads on 8.  Lengths come from the case alone, so that every seed costs the same.

The cache: keys [layer, page, head, token, dim]; values [layer, page, head, token / n, dim, n] with n values in 16 bytes.
"""
import math
import random

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2}

_ATTEND = {"op": "attend", "heads": 32, "kv_heads": 32, "dim": 128, "page": 16, "dtype": "f16", "batch": 1, "tokens": 1, "length": 2048,
           "ragged": False, "empty": False, "window": 0, "tree": False, "starts": False, "mix": 1}
_APPEND = {"op": "append", "heads": 32, "kv_heads": 32, "dim": 128, "page": 16, "dtype": "f16", "batch": 1, "tokens": 1, "length": 2048,
           "ragged": False, "empty": False, "norm": "none", "rotary": "half", "rotary_dim": 128, "scaling": "plain", "mix": 1}
_PAGES = {"op": "pages", "kind": "verify", "layers": 32, "kv_heads": 8, "dim": 128, "page": 16, "dtype": "f16", "batch": 16, "tokens": 5,
          "length": 1024, "mix": 1}


def _case(base, name, **changes):
    c = dict(base, name=name)
    c.update(changes)
    return c


def listed():
    return [
        # the first tokens of one stream: what a call costs when there is little data
        _case(_ATTEND, "attend_short", length=77),
        # one stream of an OPT-6.7B- or Llama-2-7B-shaped layer with a full context
        _case(_ATTEND, "attend_one_stream", length=2048),
        # eight streams of a Falcon-7B-shaped layer, 71 query heads on one key head, lengths as they come
        _case(_ATTEND, "attend_one_key_head", heads=71, kv_heads=1, dim=64, batch=8, length=2047, ragged=True, mix=3),
        # verification of five tokens per sequence, drafted as a tree, shared key heads, one sequence not in use
        _case(_ATTEND, "attend_verify_tree", kv_heads=8, dtype="bf16", batch=16, tokens=5, length=6001, ragged=True, empty=True, tree=True,
              page=32, mix=4),
        # one sequence with a very long context
        _case(_ATTEND, "attend_long", kv_heads=8, dtype="bf16", length=200003, page=64),
        # a full serving batch
        _case(_ATTEND, "attend_batch", kv_heads=8, batch=64, length=8192, ragged=True, mix=6),
        # a Phi-2-shaped layer in fp32, a sliding window, left padding
        _case(_ATTEND, "attend_window_f32", dim=80, dtype="f32", batch=8, length=1999, ragged=True, window=1000, starts=True, mix=7),
        # one new token of one stream, Llama-2-7B-shaped
        _case(_APPEND, "append_token"),
        # prompts in pieces of up to 64 tokens, Persimmon-8B-shaped: normalised queries and keys, half of the head rotated
        _case(_APPEND, "append_prompt", heads=64, kv_heads=64, dim=64, dtype="bf16", batch=32, tokens=64, length=901, norm="layer",
              rotary_dim=32, ragged=True, mix=5),
        # drafted tokens that are all rejected: pages taken and given back, no data moved
        _case(_PAGES, "pages_verify", layers=2, batch=64, length=2000),
        # eight beams of each of four prompts
        _case(_PAGES, "pages_fork", kind="fork", kv_heads=32, batch=4, tokens=8, length=300),
        # a burst of sequences, half of them end, the pool is made dense again
        _case(_PAGES, "pages_burst", kind="burst", batch=24, length=700, mix=2),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """A cache of any of the head layouts and types, driven in any of the ways above, from one token to long contexts."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["attend", "attend", "attend", "append", "append", "pages"])
        heads, kv_heads, dim = rng.choice([(32, 32, 128), (71, 1, 64), (32, 32, 80), (64, 64, 64), (32, 8, 128), (16, 2, 128), (24, 8, 96),
                                           (16, 4, 256), (12, 12, 64), (20, 5, 112), (8, 1, 32)])
        c = dict({"attend": _ATTEND, "append": _APPEND, "pages": _PAGES}[op], kv_heads=kv_heads, dim=dim,
                 page=rng.choice([16, 16, 32, 64, 128]), dtype=rng.choice(["f16", "f16", "bf16", "bf16", "f32"]), mix=rng.randint(1, 10 ** 6))
        if op == "attend":
            c.update(heads=heads, batch=_log(rng, 1, 128), tokens=rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 64)]),
                     length=_log(rng, 1, 200000), ragged=rng.random() < 0.7, empty=rng.random() < 0.2, starts=rng.random() < 0.2)
            if rng.random() < 0.25:
                c["window"] = _log(rng, 16, 8192)
            c["tree"] = 1 < c["tokens"] and rng.random() < 0.4
        elif op == "append":
            c.update(heads=heads, batch=_log(rng, 1, 128), tokens=rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 128)]),
                     length=_log(rng, 1, 100000), ragged=rng.random() < 0.6, empty=rng.random() < 0.2,
                     norm=rng.choice(["none", "rms", "layer"]), rotary=rng.choice(["half", "interleaved"]),
                     rotary_dim=rng.choice([0] + [r for r in (16, 32, 64, 80, 96, 112, 128, 256) if r <= dim] * 2),
                     scaling=rng.choice(["plain", "plain", "linear", "base", "ramp"]))
        else:
            c.update(kind=rng.choice(["verify", "fork", "burst"]), layers=_log(rng, 1, 32), batch=_log(rng, 1, 64),
                     tokens=rng.randint(1, 8), length=_log(rng, 1, 4000))
        if _cost(c) <= most and _cache_bytes(c) <= (4 << 30 if op == "attend" else 2 << 30):
            return c


def _cost(c):
    """Something like time: bytes at the rate of a copy, operations at that of plain products in 32 bits, calls."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 4e13 + 2e-6 * c["batch"]


def _rows(c):
    """Per row of the batch: cached tokens, new ones among them, first visible one."""
    rng = random.Random(c["mix"])
    lengths, fresh, starts = [], [], []
    for i in range(c["batch"]):
        n, f = c["length"], c["tokens"]
        if c["ragged"] and i:
            n, f = _log(rng, max(1, n // 16), n), rng.randint(1, f)
        if c["empty"] and i == c["batch"] // 2:
            n, f = 0, 0
        n, f = (max(n, f), f) if c["op"] == "append" else (n, min(n, f))
        lengths.append(n)
        fresh.append(f)
        starts.append(rng.randint(0, n // 4) if c.get("starts") else 0)
    return lengths, fresh, starts


def _sequence_lengths(c):
    rng = random.Random(c["mix"])
    return [_log(rng, max(1, c["length"] // 8), c["length"]) for _ in range(c["batch"])]


def _pages_of(c, lengths):
    return [-(-n // c["page"]) for n in lengths]


def _pool(c):
    """Sequences, pages of the pool, pages of a sequence at most."""
    if c["op"] != "pages":
        per = _pages_of(c, _rows(c)[0])
        return c["batch"] + 1, sum(per) + 3, max(per) + 1
    lengths = _sequence_lengths(c)
    if c["kind"] == "verify":
        per = _pages_of(c, [n + c["tokens"] for n in lengths])
        return c["batch"], sum(per), max(per)
    per = _pages_of(c, lengths)
    if c["kind"] == "fork":
        return c["batch"] * (1 + c["tokens"]), sum(per) + c["batch"] * c["tokens"], max(per)
    return c["batch"], sum(per) + 1, max(per)


def _page_bytes(c):
    """Of one page of the keys of one layer."""
    return c["kv_heads"] * c["page"] * c["dim"] * _SIZE[c["dtype"]]


def _cache_bytes(c):
    return 2 * c.get("layers", 1) * _pool(c)[1] * _page_bytes(c)


def work(case):
    c, e = case, _SIZE[case["dtype"]]
    if c["op"] == "attend":
        read, seen, rows = 0, 0, 0
        for n, f, start in zip(*_rows(c)):
            read += max(0, n - max(start, n - f + 1 - c["window"] if c["window"] else 0)) if f else 0
            for t in range(f):
                last = n - f + t
                seen += max(0, last + 1 - max(start, last + 1 - c["window"] if c["window"] else 0))
            rows += f
        table = 4 * -(-read // c["page"])
        return {"bytes": 2 * read * c["kv_heads"] * c["dim"] * e + rows * c["heads"] * c["dim"] * e + table +
                c["batch"] * c["tokens"] * c["heads"] * c["dim"] * e, "flops": 4 * seen * c["heads"] * c["dim"]}
    if c["op"] == "append":
        rows = sum(_rows(c)[1])
        values = (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        rotated = (c["heads"] + c["kv_heads"]) * c["rotary_dim"]
        normed = (c["heads"] + c["kv_heads"]) * c["dim"] * {"none": 0, "rms": 4, "layer": 7}[c["norm"]]
        return {"bytes": rows * values * e + (rows * 2 * c["kv_heads"] + c["batch"] * c["tokens"] * c["heads"]) * c["dim"] * e,
                "flops": rows * (3 * rotated + normed)}
    seqs, pages, _ = _pool(c)
    lengths = _sequence_lengths(c)
    per = _pages_of(c, lengths)
    if c["kind"] == "verify":
        copied, entries = 0, sum(_pages_of(c, [n + c["tokens"] for n in lengths])) - sum(per)
    elif c["kind"] == "fork":
        copied, entries = c["tokens"] * sum(n % c["page"] != 0 for n in lengths), c["tokens"] * sum(per)
    else:
        live = sum(per[0::2])
        held, at = [], 0
        for i, p in enumerate(per):
            held += list(range(at, at + p)) if i % 2 == 0 else []
            at += p
        copied, entries = sum(p >= live for p in held), sum(per)
    return {"bytes": copied * 4 * c["layers"] * _page_bytes(c) + 16 * entries + 12 * seqs, "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _frequencies(c):
    """Angle per position of every rotated pair, and the factor on what is rotated."""
    r, base, factor, trained = c["rotary_dim"], 10000.0, 4.0, 2048
    if c["scaling"] == "base" and r > 2:
        base *= factor ** (r / (r - 2.0))
    f = [base ** (-2.0 * i / r) for i in range(r // 2)]
    if c["scaling"] == "linear":
        f = [v / factor for v in f]
    if c["scaling"] == "ramp":                            # by the turns a pair makes over the trained length
        keep = [min(1.0, max(0.0, (trained * v / (2 * math.pi) - 1.0) / (32.0 - 1.0))) for v in f]
        f = [k * v + (1.0 - k) * v / factor for k, v in zip(keep, f)]
    return f, 0.1 * math.log(factor) + 1.0 if c["scaling"] == "ramp" else 1.0


def _inputs(c, seed):
    """Everything but the cache's two large arrays, from the seed."""
    host, gen = random.Random(seed), torch.Generator(device="cuda")
    gen.manual_seed(seed)
    seqs, pages, width = _pool(c)
    s = {"case": c, "seqs": seqs, "pages": pages, "width": width, "gen": gen, "dtype": _TYPES[c["dtype"]]}
    gpu = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    if c["op"] == "pages":
        s["lengths"] = _sequence_lengths(c)
        if c["kind"] == "verify":                         # (which of a burst's sequences end decides how many pages move)
            host.shuffle(s["lengths"])
        return s
    lengths, fresh, starts = _rows(c)
    slots = list(range(seqs))
    host.shuffle(slots)
    slots = slots[:c["batch"]]
    free = list(range(pages))
    host.shuffle(free)
    table, of_slot, fresh_of_slot = [[-1] * width for _ in range(seqs)], [0] * seqs, [0] * seqs
    for slot, n, f in zip(slots, lengths, fresh):
        for j in range(-(-n // c["page"])):
            table[slot][j] = free.pop()
        of_slot[slot], fresh_of_slot[slot] = n, f
    s.update(lengths=lengths, fresh=fresh, slots=slots, slots_gpu=gpu(slots), table=gpu(table), lengths_gpu=gpu(of_slot),
             fresh_gpu=gpu(fresh_of_slot))
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    b, t, h, kvh, d = c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["dim"]
    if c["op"] == "attend":
        s["q"] = (1.5 * rand(b, t, h, d)).to(s["dtype"])
        s["starts"] = starts if c["starts"] else None
        s["starts_gpu"] = gpu(starts) if c["starts"] else None
        s["tree"] = None
        if c["tree"]:                                     # a word per new token: itself and the tokens it was drafted after
            s["tree"] = []
            for i in range(b):
                words = []
                for j in range(t):
                    words.append((words[host.randrange(j)] if j else 0) | 1 << j)
                s["tree"].append(words)
            s["tree_gpu"] = torch.tensor([[w - (1 << 64) if w >> 63 else w for w in ws] for ws in s["tree"]], dtype=torch.int64, device="cuda")
    else:
        # one row of queries, keys and values per token, as a fused projection leaves them
        qkv = rand(b, t, (h + 2 * kvh) * d).to(s["dtype"])
        s["q"] = qkv[..., :h * d].view(b, t, h, d)
        s["k_new"] = qkv[..., h * d:(h + kvh) * d].view(b, t, kvh, d)
        s["v_new"] = qkv[..., (h + kvh) * d:].view(b, t, kvh, d)
        s["norm"] = None
        if c["norm"] != "none":
            s["norm"] = [1.0 + 0.1 * rand(d), 0.1 * rand(d), 1.0 + 0.1 * rand(d), 0.1 * rand(d)]
            if c["norm"] == "rms":
                s["norm"][1] = s["norm"][3] = None
        s["frequencies"], s["magnitude"] = _frequencies(c)
    return s


_EPS = 1e-5


def _shapes(c, pages):
    n = 16 // _SIZE[c["dtype"]]
    head = (c.get("layers", 1), pages, c["kv_heads"])
    return head + (c["page"], c["dim"]), head + (c["page"] // n, c["dim"], n)


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    if own:
        import paper_2312_11514_amd as lif
        extra = {}
        if c["op"] == "append":
            extra = {"norm": {"none": lif.NORM_NONE, "rms": lif.NORM_RMS, "layer": lif.NORM_LAYER}[c["norm"]], "norm_eps": _EPS,
                     "rotary": lif.ROTARY_HALF if c["rotary"] == "half" else lif.ROTARY_INTERLEAVED, "rotary_dim": c["rotary_dim"],
                     "rotary_scale": s["magnitude"]}
            if c["rotary_dim"]:
                extra["frequencies"] = torch.tensor(s["frequencies"], dtype=torch.float64, device="cuda")
        kv = s["kv"] = lif.KVCache(layers=c.get("layers", 1), heads=c.get("heads", c["kv_heads"]), kv_heads=c["kv_heads"], head_dim=c["dim"],
                                   page_tokens=c["page"], pages=s["pages"], max_seqs=s["seqs"], max_pages=s["width"],
                                   max_tokens=c["tokens"], dtype=c["dtype"], **extra)
        s["k"], s["v"] = kv.k, kv.v
    else:
        ks, vs = _shapes(c, s["pages"])
        s["k"], s["v"] = torch.empty(ks, dtype=s["dtype"], device="cuda"), torch.empty(vs, dtype=s["dtype"], device="cuda")
    s["k"].normal_(generator=s["gen"])
    s["v"].normal_(generator=s["gen"])
    if c["op"] == "pages":
        _prepare_pages(s)
        return s
    if own:
        kv.table.copy_(s["table"])
        kv.lengths.copy_(s["lengths_gpu"])
        kv.fresh.copy_(s["fresh_gpu"])
        kv.adopt()
    elif c["op"] == "append" and c["rotary_dim"]:         # cosines and sines by position, as such a program keeps them
        at = torch.arange(max(1, c["length"], c["tokens"]), dtype=torch.float64, device="cuda")[:, None]
        angle = at * torch.tensor(s["frequencies"], dtype=torch.float64, device="cuda")
        s["cos"], s["sin"] = (s["magnitude"] * angle.cos()).float(), (s["magnitude"] * angle.sin()).float()
    s["out"] = torch.empty_like(s["q"], memory_format=torch.contiguous_format)
    return s


def _prepare_pages(s):
    c = s["case"]
    gpu = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    if not own:
        s["table"] = torch.full((s["seqs"], s["width"]), -1, dtype=torch.int32, device="cuda")
        s["lengths_gpu"], s["fresh_gpu"] = gpu([0] * s["seqs"]), gpu([0] * s["seqs"])
        s["refs"] = gpu([0] * s["pages"])
    reserve = s["kv"].reserve if own else lambda counts: _reserve(s, counts)
    b, lengths = c["batch"], s["lengths"]
    if c["kind"] == "verify":
        reserve(gpu(lengths))
        s["counts"], s["back"] = gpu([c["tokens"]] * b), gpu(lengths)
    elif c["kind"] == "fork":
        copies = b * c["tokens"]
        reserve(gpu(lengths + [0] * copies))
        s["back"] = gpu([-1] * b + [0] * copies)
        s["src"] = gpu([i for i in range(b) for _ in range(c["tokens"])])
        s["dst"] = gpu(list(range(b, b + copies)))
    else:
        s["none"], s["counts"], s["back"] = gpu([0] * b), gpu(lengths), gpu([-1 if i % 2 == 0 else 0 for i in range(b)])


# ---- one pass ----------------------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if c["op"] == "attend":
        if own:
            s["kv"].attend(0, s["q"], s["out"], window=c["window"], starts=s["starts_gpu"], tree=s["tree_gpu"] if s["tree"] else None,
                           slots=s["slots_gpu"])
            return s["out"]
        return _attend(s)
    if c["op"] == "append":
        if own:
            s["kv"].append(0, s["q"], s["k_new"], s["v_new"], s["out"], norm=s["norm"], slots=s["slots_gpu"])
            return {"q": s["out"], "k": s["k"], "v": s["v"]}
        return _append(s)
    if own:
        kv = s["kv"]
        if c["kind"] == "verify":
            kv.reserve(s["counts"])
            kv.truncate(s["back"])
        elif c["kind"] == "fork":
            kv.truncate(s["back"])
            kv.fork(s["src"], s["dst"])
        else:
            kv.truncate(s["none"])
            kv.reserve(s["counts"])
            kv.truncate(s["back"])
            kv.compact()
        held = {"table": kv.table, "lengths": kv.lengths, "refs": kv.refs}
    else:
        if c["kind"] == "verify":
            _reserve(s, s["counts"])
            _truncate(s, s["back"])
        elif c["kind"] == "fork":
            _truncate(s, s["back"])
            _fork(s, s["src"].long(), s["dst"].long())
        else:
            _truncate(s, s["none"])
            _reserve(s, s["counts"])
            _truncate(s, s["back"])
            _compact(s)
        held = {"table": s["table"], "lengths": s["lengths_gpu"], "refs": s["refs"]}
    return held if c["kind"] == "verify" else dict(held, k=s["k"], v=s["v"])


# ---- the operators in their plain form ---------------------------------------------------------------------------------------

def _attend(s):
    c = s["case"]
    h, kvh, d, page, t = c["heads"], c["kv_heads"], c["dim"], c["page"], c["tokens"]
    group, out = h // kvh, torch.zeros_like(s["out"])
    for i, (slot, n, f) in enumerate(zip(s["slots"], s["lengths"], s["fresh"])):
        if f == 0:
            continue
        start = s["starts"][i] if s["starts"] else 0
        low = max(start, n - f + 1 - c["window"] if c["window"] else 0) // page
        pages = s["table"][slot, low:-(-n // page)].long()
        keys = s["k"][0, pages].permute(1, 0, 2, 3).reshape(kvh, -1, d).float()
        values = s["v"][0, pages].permute(1, 0, 2, 4, 3).reshape(kvh, -1, d).float()
        q = s["q"][i, :f].float().view(f, kvh, group, d).permute(1, 0, 2, 3).reshape(kvh, f * group, d)
        at = low * page + torch.arange(keys.shape[1], device="cuda")
        new = at - (n - f)                                # which of the new tokens, negative: an older one
        token = torch.arange(f, device="cuda")[:, None]
        if s["tree"]:
            seen = (new < 0) | ((s["tree_gpu"][i, :f, None] >> new.clamp(0, 63)) & 1 == 1)
        else:
            seen = new <= token
        seen = seen & (at >= start) & (at < n)
        if c["window"]:
            seen = seen & (new > token - c["window"])
        score = torch.matmul(q, keys.transpose(1, 2)) * (1.0 / math.sqrt(d))
        score = score.view(kvh, f, group, -1).masked_fill(~seen[None, :, None, :], -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = e.sum(-1, keepdim=True)
        o = torch.matmul(e.view(kvh, f * group, -1), values).view(kvh, f, group, d)
        o = torch.where(total > 0, o / total, torch.zeros_like(o))
        out[i, :f] = o.permute(1, 0, 2, 3).reshape(f, h, d).to(s["dtype"])
    return out


def _norm_plain(c, x, w, b):
    if c["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS) * w
    return x + b if c["norm"] == "layer" else x


def _rotate_plain(c, x, cos, sin):
    r = c["rotary_dim"]
    if r == 0:
        return x
    if c["rotary"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([y, x[..., r:]], -1)


def _append(s):
    c = s["case"]
    slots, page, e = s["slots_gpu"].long(), c["page"], 16 // _SIZE[c["dtype"]]
    n, f = s["lengths_gpu"][slots].long()[:, None], s["fresh_gpu"][slots].long()[:, None]
    t = torch.arange(c["tokens"], device="cuda")[None, :]
    there, at = t < f, (n - f + t).clamp(min=0)
    q, k, v = s["q"].float(), s["k_new"].float(), s["v_new"]
    if s["norm"] is not None:
        q, k = _norm_plain(c, q, s["norm"][0], s["norm"][1]), _norm_plain(c, k, s["norm"][2], s["norm"][3])
    if c["rotary_dim"]:
        at_table = at.clamp(max=s["cos"].shape[0] - 1)
        cos, sin = s["cos"][at_table][:, :, None, :], s["sin"][at_table][:, :, None, :]
        q, k = _rotate_plain(c, q, cos, sin), _rotate_plain(c, k, cos, sin)
    out = torch.where(there[:, :, None, None], q, torch.zeros_like(q)).to(s["dtype"])
    row, token = there.nonzero(as_tuple=True)
    where = at[row, token]
    pages, offset = s["table"][slots[row], where // page].long(), where % page
    s["k"][0][pages, :, offset] = k[row, token].to(s["dtype"])
    s["v"][0][pages, :, offset // e, :, offset % e] = v[row, token]
    return {"q": out, "k": s["k"], "v": s["v"]}


def _reserve(s, counts):
    page, table = s["case"]["page"], s["table"]
    had, needs = -(-s["lengths_gpu"] // page), -(-(s["lengths_gpu"] + counts) // page)
    first = (needs - had).cumsum(0) - (needs - had)
    order = torch.argsort((s["refs"] > 0).int(), stable=True)          # the free pages first, lowest numbers first
    column = torch.arange(table.shape[1], device="cuda")[None, :]
    fill = (column >= had[:, None]) & (column < needs[:, None])
    got = order[(first[:, None] + column - had[:, None]).clamp(0, len(order) - 1)]
    s["table"] = torch.where(fill, got.int(), table)
    s["refs"] = s["refs"].scatter_add(0, got.flatten(), fill.flatten().int())
    s["lengths_gpu"], s["fresh_gpu"] = s["lengths_gpu"] + counts, counts


def _truncate(s, to):
    page, table = s["case"]["page"], s["table"]
    new = torch.where(to < 0, s["lengths_gpu"], torch.minimum(to, s["lengths_gpu"]))
    column = torch.arange(table.shape[1], device="cuda")[None, :]
    drop = (column >= -(-new // page)[:, None]) & (column < -(-s["lengths_gpu"] // page)[:, None])
    s["refs"] = s["refs"].scatter_add(0, table.clamp(min=0).flatten().long(), -drop.flatten().int())
    s["table"] = torch.where(drop, torch.full_like(table, -1), table)
    s["lengths_gpu"], s["fresh_gpu"] = new, torch.zeros_like(new)


def _fork(s, src, dst):
    page, rows = s["case"]["page"], s["table"][src]
    n = s["lengths_gpu"][src]
    held, partial = -(-n // page), n % page != 0
    order = torch.argsort((s["refs"] > 0).int(), stable=True)
    rank = partial.long().cumsum(0) - partial.long()
    column = torch.arange(rows.shape[1], device="cuda")[None, :]
    is_last = (column == (held - 1)[:, None]) & partial[:, None]
    old = rows.gather(1, (held - 1).clamp(min=0).long()[:, None])[:, 0]
    new = torch.where(partial, order[rank].int(), old)
    s["k"][:, new.long()] = s["k"][:, old.long()]
    s["v"][:, new.long()] = s["v"][:, old.long()]
    rows = torch.where(is_last, new[:, None], torch.where(column < held[:, None], rows, torch.full_like(rows, -1)))
    s["table"][dst] = rows
    s["refs"] = s["refs"].scatter_add(0, rows.clamp(min=0).flatten().long(), (rows >= 0).flatten().int())
    s["lengths_gpu"][dst] = n
    s["fresh_gpu"][dst] = 0


def _compact(s):
    used = s["refs"] > 0
    live, ids = used.sum(), torch.arange(len(used), device="cuda")
    holes = (~used & (ids < live)).nonzero()[:, 0]
    movers = (used & (ids >= live)).nonzero()[:, 0].flip(0)
    s["k"][:, holes] = s["k"][:, movers]
    s["v"][:, holes] = s["v"][:, movers]
    to = ids.int()
    to[movers] = holes.int()
    s["table"] = torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], s["table"])
    refs = s["refs"].clone()
    refs[holes] = s["refs"][movers]
    refs[movers] = 0
    s["refs"] = refs


# ---- the operators by their definition, in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None                                       # whole numbers and copies
    s = _inputs(c, seed)
    ks, vs = _shapes(c, s["pages"])
    s["k"], s["v"] = torch.empty(ks, dtype=s["dtype"], device="cuda"), torch.empty(vs, dtype=s["dtype"], device="cuda")
    s["k"].normal_(generator=s["gen"])
    s["v"].normal_(generator=s["gen"])
    return _exact_attend(s) if c["op"] == "attend" else _exact_append(s)


def _exact_attend(s):
    c = s["case"]
    if sum(f * n for f, n in zip(s["fresh"], s["lengths"])) * c["heads"] > 4e8 or c["batch"] * c["kv_heads"] > 4096:
        return None
    group, page = c["heads"] // c["kv_heads"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    table = s["table"].tolist()
    for i, slot in enumerate(s["slots"]):
        n, f = s["lengths"][i], s["fresh"][i]
        if f == 0:
            continue
        pages = torch.tensor(table[slot][:-(-n // page)], device="cuda")
        seen = torch.zeros(f, n, dtype=torch.bool)
        for t in range(f):
            seen[t, s["starts"][i] if s["starts"] else 0:n - f] = True
            for u in range(f):
                old = n - f + u < (s["starts"][i] if s["starts"] else 0)
                seen[t, n - f + u] = not old and bool(s["tree"][i][t] >> u & 1 if s["tree"] else u <= t)
            if c["window"]:
                seen[t, :max(0, n - f + t + 1 - c["window"])] = False
        seen = seen.cuda()
        for g in range(c["kv_heads"]):
            keys = s["k"][0, pages, g].double().reshape(-1, c["dim"])[:n]
            values = s["v"][0, pages, g].double().transpose(2, 3).reshape(-1, c["dim"])[:n]
            for t in range(f):
                at = seen[t].nonzero()[:, 0]
                if len(at) == 0:
                    continue
                dots = s["q"][i, t, g * group:(g + 1) * group].double() @ keys[at].T.contiguous() / math.sqrt(c["dim"])
                weight = torch.exp(dots - dots.max(1, keepdim=True)[0])
                out[i, t, g * group:(g + 1) * group] = (weight / weight.sum(1, keepdim=True)) @ values[at]
    return out


def _exact_append(s):
    c = s["case"]
    if 16 * s["k"].numel() > 16 << 30:
        return None
    r, page, e = c["rotary_dim"], c["page"], 16 // _SIZE[c["dtype"]]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    k, v = s["k"].double(), s["v"].double()
    frequency = torch.tensor(s["frequencies"], dtype=torch.float64, device="cuda")
    table = s["table"].tolist()

    def formula(x, weight, bias, positions):
        x = x.double()
        if weight is not None:
            mean = x.mean(-1, keepdim=True) if c["norm"] == "layer" else 0.0
            x = (x - mean) * ((x - mean) ** 2).mean(-1, keepdim=True).add(_EPS).rsqrt() * weight.double()
            x = x if bias is None else x + bias.double()
        if r:
            turn = torch.polar(torch.full((1,), s["magnitude"], dtype=torch.float64, device="cuda"), positions[:, None] * frequency)[:, None]
            pairs = (x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if c["rotary"] == "half" else x[..., :r].unflatten(-1, (r // 2, 2)))
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            turned = turned.transpose(-1, -2) if c["rotary"] == "half" else turned
            x = torch.cat([turned.flatten(-2), x[..., r:]], -1)
        return x

    wq, bq, wk, bk = s["norm"] or [None] * 4
    for i, slot in enumerate(s["slots"]):
        n, f = s["lengths"][i], s["fresh"][i]
        if f == 0:
            continue
        at = torch.arange(n - f, n, device="cuda")
        out[i, :f] = formula(s["q"][i, :f], wq, bq, at.double())
        new = formula(s["k_new"][i, :f], wk, bk, at.double())
        pages = torch.tensor(table[slot], device="cuda")[at // page]
        k[0, pages, :, at % page] = new
        v[0, pages, :, at % page // e, :, at % page % e] = s["v_new"][i, :f].double()
    return {"q": out, "k": k, "v": v}
