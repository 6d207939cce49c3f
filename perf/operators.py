"""Workloads of dense attention over packed sequences and of its learned relative position bias.

A case is one pass as a program makes it: `forward` (inference; a prompt, a cross attention, or single new tokens over a
cache of keys and values) or `train` (forward, then the gradients of everything that learns).  Sequences of different
lengths lie packed one behind the other, or, for a cache, each at the start of a slot of its own.

Formulas, for query i and key j of one sequence with Lq queries and Lk keys (query i stands at position i + Lk - Lq):
  S = scale q k^T + bias[head, bucket(j - position of i)], keys behind the query's position left out where causal,
  P = softmax(S), out = P v, and the gradients of that.
"""
import math
import random

import torch

own = False


def _case(name, kind, seqs, q_min, q_max, heads, h_kv, d, k_min=0, k_max=0, causal=False, cache=False, fused=False,
          buckets=0, max_distance=0, two_sided=True):
    """q_min .. q_max: query lengths.  k_min, k_max: key lengths of their own (0: a sequence attends to itself).  cache: keys
    lie in slots of k_max rows of which the first k_len are filled.  fused: q, k, v are slices of one projection.
    buckets: size of the bias' table (0: none), for distances that count up to max_distance, to both sides or behind only."""
    return {"name": name, "kind": kind, "seqs": seqs, "q_min": q_min, "q_max": q_max, "heads": heads, "h_kv": h_kv, "d": d,
            "k_min": k_min, "k_max": k_max, "causal": causal, "cache": cache, "fused": fused, "buckets": buckets,
            "max_distance": max_distance, "two_sided": two_sided}


def listed():
    return [
        # four streams that each take one token more, right after a short prompt: latency is all there is
        _case("serve short", "forward", 4, 1, 1, 16, 16, 64, 65, 513, True, cache=True),
        # sixteen streams of very different age, grouped heads: a step of a serving loop
        _case("serve grouped", "forward", 16, 1, 1, 16, 2, 128, 700, 12000, True, cache=True),
        # one stream over the largest scene of the repository (428 K tokens), one query: few rows, all the keys
        _case("serve one long", "forward", 1, 1, 1, 16, 2, 128, 428032, 428032, True, cache=True),
        # a few small things at once, with the bias, straight from a fused projection
        _case("small biased forward", "forward", 5, 17, 130, 4, 4, 64, fused=True, buckets=32, max_distance=128),
        # objects of a batch attend to themselves, lengths as active voxels leave them
        _case("packed forward", "forward", 6, 700, 4096, 16, 16, 64),
        # prompts with the paper's heads (32 of 32 channels on 2 key/value heads), causal
        _case("causal grouped forward", "forward", 3, 1531, 8000, 32, 2, 32, causal=True),
        # volume tokens look at image tokens: queries and keys are different sets
        _case("cross forward", "forward", 4, 1024, 4097, 8, 8, 128, 2048, 9216),
        # one long prompt at the repository's largest heads
        _case("long causal forward", "forward", 1, 16384, 16384, 16, 16, 128, causal=True),
        # a training step of the paper's heads over packed objects
        _case("grouped train", "train", 4, 333, 2500, 32, 2, 32),
        # the largest training step
        _case("long causal train", "train", 2, 4500, 8192, 16, 16, 128, causal=True),
        # a training step over many short sequences with the bias: everything is near
        _case("short biased train", "train", 7, 1, 257, 8, 4, 32, buckets=32, max_distance=128),
        # an ordinary training step with the bias, causal
        _case("biased causal train", "train", 3, 1000, 4096, 16, 8, 64, causal=True, buckets=32, max_distance=128, two_sided=False),
    ]


def _spread(n, lo, hi, start):
    """n lengths between lo and hi, the largest among them (a case's own, whatever the seed)."""
    return [hi if i == n // 2 else lo + int((hi - lo + 1) * ((start + 0.618034 * (i + 1)) % 1.0)) for i in range(n)]


def _lengths(case):
    q = _spread(case["seqs"], case["q_min"], case["q_max"], 0.0)
    k = _spread(case["seqs"], case["k_min"], case["k_max"], 0.37) if case["k_max"] else q
    return q, k


def _pairs(case):
    """visible (query, key) pairs of one head"""
    q, k = _lengths(case)
    return sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(q, k))


def _cost(case):
    return _pairs(case) * case["heads"] * (32 + case["d"]) * (4 if case["kind"] == "train" else 1)


def _padded(case):
    return case["seqs"] * case["heads"] * case["q_max"] * (case["k_max"] or case["q_max"])


def draw(rng: random.Random):
    largest = max(listed(), key=_cost)
    while True:
        d = rng.choice((32, 64, 128))
        heads = rng.choice((1, 2, 3, 4, 6, 8, 16, 32))
        h_kv = heads if rng.random() < 0.5 else rng.choice([h for h in range(1, heads + 1) if heads % h == 0 and heads // h <= 16])
        what = rng.choice(("serve", "self", "cross", "train", "train"))
        seqs = max(1, round(2 ** rng.uniform(0, 5 if what == "serve" else 3.5)))
        q_max = round(2 ** rng.uniform(3 if what == "train" else 0, 13))
        q_min = max(1, round(q_max * rng.uniform(0.05, 1.0)))
        causal, k_min, k_max = rng.random() < 0.5, 0, 0
        if what == "serve":
            q_min, q_max = 1, rng.choice((1, 1, 1, 2, 5))
            k_max = round(2 ** rng.uniform(4, 16))
            k_min = max(q_max, round(k_max * rng.uniform(0.1, 1.0)))
            causal = True
        elif what == "cross" or (what == "train" and rng.random() < 0.3):
            k_max = round(2 ** rng.uniform(3, 13))
            k_min = max(1, round(k_max * rng.uniform(0.1, 1.0)))
            causal = False
        buckets = rng.choice((0, 0, 16, 32))
        case = _case("", "train" if what == "train" else "forward", seqs, q_min, q_max, heads, h_kv, d, k_min, k_max, causal,
                     what == "serve", k_max == 0 and rng.random() < 0.3, buckets, rng.choice((32, 128)) if buckets else 0,
                     not causal or rng.random() < 0.3)
        del case["name"]
        rows = case["seqs"] * (case["q_max"] * heads + (case["k_max"] or case["q_max"]) * h_kv) * d
        if _cost(case) <= 0.5 * _cost(largest) and _padded(case) <= 2.2e9 and rows <= 2.5e8:
            return case


def _bounds(case):
    """Ascending distances j - i at which a new bucket begins.  Half of a side's buckets hold one distance each, the others grow
    geometrically up to max_distance; to the left of 0 the same mirrored.  (From the definition, by looking at every distance.)"""
    n = case["buckets"]
    side = n // 2 if case["two_sided"] else n
    exact_n = side // 2

    def bucket(distance):
        if distance < exact_n:
            return distance
        return min(side - 1, exact_n + int(math.log(distance / exact_n) / math.log(case["max_distance"] / exact_n) * (side - exact_n) + 1e-9))

    starts = [x for x in range(1, case["max_distance"] + 1) if bucket(x) != bucket(x - 1)]
    left = [1 - x for x in reversed(starts)]
    return left + ([1] + [x for x in starts if x > 1] if case["two_sided"] else [])


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16)

    q_len, k_len = _lengths(case)
    h, hk, d = case["heads"], case["h_kv"], case["d"]

    def offsets(lengths):
        return torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).to(torch.int32).to(dev)

    s = {"case": case, "q_off": offsets(q_len), "k_lens": None, "q_max": max(q_len), "k_max": max(k_len)}
    n_q = sum(q_len)
    if case["cache"]:
        s["k_off"] = offsets([case["k_max"]] * case["seqs"])
        s["k_lens"] = torch.tensor(k_len, dtype=torch.int32).to(dev)
        n_k = case["k_max"] * case["seqs"]
    else:
        s["k_off"] = offsets(k_len) if case["k_max"] else s["q_off"]
        n_k = sum(k_len)

    def rows():
        """q, k, v-like tensors: three of their own, or slices of one projection"""
        if case["fused"]:
            x = normal(n_q, h + 2 * hk, d)
            return x[:, :h], x[:, h:h + hk], x[:, h + hk:]
        return normal(n_q, h, d), normal(n_k, hk, d), normal(n_k, hk, d)

    s["q"], s["k"], s["v"] = rows()
    s["out"] = torch.empty((n_q, h, d), dtype=torch.bfloat16, device=dev)
    s["lse"] = s["bias"] = s["dbias"] = None
    s["bounds"] = []
    if case["buckets"]:
        s["bounds"] = _bounds(case)
        s["bias"] = normal(h, len(s["bounds"]) + 1)
    if case["kind"] == "train":
        s["lse"] = torch.empty((n_q, h), dtype=torch.float32, device=dev)
        s["dout"] = normal(n_q, h, d)
        s["dq"], s["dk"], s["dv"] = rows()
        if case["buckets"]:
            s["dbias"] = torch.empty_like(s["bias"])
    return s


# ---- the plain form ---------------------------------------------------------------------------------------------------
def _to_batch(x, start, width):
    """rows of every sequence, in 32 bits, side by side: [seqs, heads, width, d] (rows past a sequence's end are some other row)"""
    at = start[:, None] + torch.arange(width, device=x.device)
    return x[at.clamp(max=x.shape[0] - 1)].float().transpose(1, 2)


def _from_batch(x, offsets, n):
    """the packed rows back: [seqs, heads, width, d] -> [n, heads, d]"""
    row = torch.arange(n, device=x.device)
    seq = torch.searchsorted(offsets[1:].long(), row, right=True)
    return x.transpose(1, 2)[seq, row - offsets[seq].long()]


def _plain_pass(s):
    case = s["case"]
    h, hk, d = case["heads"], case["h_kv"], case["d"]
    q0, k0 = s["q_off"][:-1].long(), s["k_off"][:-1].long()
    q_len = s["q_off"].diff().long()
    k_len = s["k_off"].diff().long() if s["k_lens"] is None else s["k_lens"].long()
    wq, wk, n = s["q_max"], s["k_max"], case["seqs"]
    scale = 1.0 / math.sqrt(d)

    def grouped(x):  # query heads of one key/value head behind each other, so that they share a product
        return x.reshape(n, hk, (h // hk) * wq, d)

    i, j = torch.arange(wq, device=q0.device)[:, None], torch.arange(wk, device=q0.device)
    rel = j - (i + (k_len - q_len)[:, None, None])                                   # [seqs, wq, wk]
    seen = (i < q_len[:, None, None]) & (j < k_len[:, None, None])
    if case["causal"]:
        seen &= rel <= 0
    q, k, v = grouped(_to_batch(s["q"], q0, wq)), _to_batch(s["k"], k0, wk), _to_batch(s["v"], k0, wk)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(n, h, wq, wk)
    if s["bias"] is not None:
        bucket = torch.bucketize(rel, torch.tensor(s["bounds"], device=rel.device), right=True)
        p += s["bias"].float()[:, bucket].transpose(0, 1)
    p.masked_fill_(~seen[:, None], -math.inf)
    top = p.amax(3, keepdim=True).clamp(min=-3e38)
    p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    p /= total.clamp(min=1e-38)
    out = torch.matmul(p.view(n, hk, -1, wk), v).view(n, h, wq, d)
    n_q, n_k = s["q"].shape[0], s["k"].shape[0]
    result = [_from_batch(out, s["q_off"], n_q).to(torch.bfloat16)]
    if case["kind"] == "forward":
        return result
    result.append(_from_batch(torch.log(total) + top, s["q_off"], n_q)[:, :, 0])
    dout = _to_batch(s["dout"], q0, wq)
    delta = (dout * out).sum(3, keepdim=True)
    dout = grouped(dout)
    dv = torch.matmul(p.view(n, hk, -1, wk).transpose(2, 3).contiguous(), dout)
    ds = torch.matmul(dout, v.transpose(2, 3).contiguous()).view(n, h, wq, wk).sub_(delta).mul_(p)
    g = ds.view(n, hk, -1, wk)
    dq = torch.matmul(g, k).mul_(scale).view(n, h, wq, d)
    dk = torch.matmul(g.transpose(2, 3).contiguous(), q).mul_(scale)
    result += [_from_batch(dq, s["q_off"], n_q).to(torch.bfloat16), _from_batch(dk, s["k_off"], n_k).to(torch.bfloat16),
               _from_batch(dv, s["k_off"], n_k).to(torch.bfloat16)]
    if s["bias"] is not None:
        # a row's keys of one bucket lie side by side: their sum is a difference of two running sums (in 64 bits)
        running = ds.cumsum(3, dtype=torch.float64)
        place = (i + (k_len - q_len)[:, None, None])[:, None]                        # [seqs, 1, wq, 1]
        ends = torch.tensor(s["bounds"], device=q.device) + place                    # keys before these lie in lower buckets
        below = running.gather(3, (ends.clamp(1, wk) - 1).expand(n, h, wq, -1)) * (ends > 0)
        below = torch.cat([torch.zeros_like(running[..., :1]), below, running[..., -1:]], 3)
        result.append(below.diff(dim=3).sum((0, 2)).to(torch.bfloat16))
    return result


# ---- the framework's calls --------------------------------------------------------------------------------------------
def _own_pass(s):
    from paper_2604_05182_amd import binding as B
    case = s["case"]
    if "plan" not in s:  # what a program keeps: the problem's description and the workspaces
        s["plan"] = B.make_attn_params(s["q"], s["k"], s["v"], s["q_off"], s["k_off"], k_lens=s["k_lens"], causal=case["causal"],
                                       bucket_bounds=s["bounds"] if case["buckets"] else None)
        s["ws"] = B.alloc_attn_workspace(s["plan"], B.LSRM_WS_FORWARD)
        if case["kind"] == "train":
            s["ws_back"] = B.alloc_attn_workspace(s["plan"], B.LSRM_WS_BACKWARD)
    p = s["plan"]
    B.lsrm_attn_forward(p, s["q"], s["k"], s["v"], s["out"], s["lse"], s["ws"], bias=s["bias"])
    if case["kind"] == "forward":
        return [s["out"]]
    B.lsrm_attn_backward(p, s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], s["ws_back"],
                         bias=s["bias"], dbias=s["dbias"])
    return [s["out"], s["lse"], s["dq"], s["dk"], s["dv"]] + ([s["dbias"]] if case["buckets"] else [])


def run(state):
    return _own_pass(state) if own else _plain_pass(state)


def work(case):
    """q, k, v and what goes with them read once, outputs written once; two contractions a visible pair forward, five backward."""
    q, k = (sum(x) for x in _lengths(case))
    h, hk, d = case["heads"], case["h_kv"], case["d"]
    table = 2 * h * case["buckets"]
    total = 2 * d * (2 * q * h + 2 * k * hk) + table
    flops = 4.0 * d * h * _pairs(case)
    if case["kind"] == "train":
        total += 4 * q * h + 2 * d * (2 * q * h + 2 * k * hk) + table
        flops *= 3.5
    return {"bytes": float(total), "flops": flops}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    """Sequence by sequence and head by head, from the definition."""
    s = prepare(case, seed)
    train, h, hk, d = case["kind"] == "train", case["heads"], case["h_kv"], case["d"]
    q_len, k_len = _lengths(case)
    q_off, k_off = s["q_off"].tolist(), s["k_off"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in "qkv")
    db = None if s["bias"] is None else torch.zeros(s["bias"].shape, dtype=torch.float64, device="cuda")
    edges = torch.tensor(s["bounds"], device="cuda")
    for n, (lq, lk) in enumerate(zip(q_len, k_len)):
        place = torch.arange(lq, device="cuda")[:, None] + (lk - lq)
        gap = torch.arange(lk, device="cuda")[None, :] - place
        which = sum((gap >= e).long() for e in edges) if len(edges) else torch.zeros_like(gap)
        a, b = slice(q_off[n], q_off[n] + lq), slice(k_off[n], k_off[n] + lk)
        for t in range(h):
            kv = t // (h // hk)
            qh, kh, vh = s["q"][a, t].double(), s["k"][b, kv].double(), s["v"][b, kv].double()
            x = qh @ kh.T / math.sqrt(d)
            if s["bias"] is not None:
                x = x + s["bias"][t].double()[which]
            if case["causal"]:
                x = torch.where(gap > 0, float("-inf"), x)
            z = torch.logsumexp(x, 1)
            w = torch.exp(x - z[:, None])
            del x
            out[a, t], lse[a, t] = w @ vh, z
            if train:
                gh = s["dout"][a, t].double()
                dv[b, kv] += w.T @ gh
                c = w * (gh @ vh.T - (gh * out[a, t]).sum(1, keepdim=True))
                dq[a, t] = c @ kh / math.sqrt(d)
                dk[b, kv] += c.T @ qh / math.sqrt(d)
                if db is not None:
                    db[t] += torch.bincount(which.reshape(-1), c.reshape(-1), minlength=db.shape[1])
    if not train:
        return [out]
    return [out, lse, dq, dk, dv] + ([db] if db is not None else [])
