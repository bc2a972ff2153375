"""Operators around the verification pass, as timed cases: a paged key-value cache (append, attention of one new
token), probabilities from logits, and acceptance of a draft tree by given random numbers.

A case is one call of one operator, in its plain form (elementary torch operations) or through the framework
(`own = True`):

  append  new tokens' keys rotated and written to a paged cache with their values, queries rotated
  attend  attention of one new token per sequence over a paged cache; `window` keys and `sink` first ones visible,
          or all (window 0)
  probs   softmax of logits at a temperature
  accept  walk down a draft tree by acceptance tests against the target's probabilities, then a draw from what is left

Sizes: the 7B shape of the benchmark (32 heads of 128, 32000 tokens, 256 action tokens, 60-node trees, prefix 280), the
float32 reference model's heads of 64, and generic ones for grouped heads, long caches and large vocabularies.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
ACTIONS = 256


def _append(name, dtype="bf16", heads=32, kv=8, d=128, page=64, seqs=1, new=1, lo=0, hi=280, pad=0):
    """`seqs` sequences get `new` tokens each behind lo .. hi earlier ones; `pad` rows of the batch are padding."""
    return {"name": name, "kind": "append", "dtype": dtype, "heads": heads, "kv": kv, "d": d, "page": page, "seqs": seqs,
            "new": new, "lo": lo, "hi": hi, "pad": pad, "theta": 1e4}


def _attend(name, dtype="bf16", heads=32, kv=8, d=128, page=64, seqs=1, lo=280, hi=280, window=0, sink=0):
    """`seqs` sequences of lo .. hi tokens, the new one included."""
    return {"name": name, "kind": "attend", "dtype": dtype, "heads": heads, "kv": kv, "d": d, "page": page, "seqs": seqs,
            "lo": lo, "hi": hi, "window": window, "sink": sink}


def _probs(name, rows, vocab, temperature=1.0):
    return {"name": name, "kind": "probs", "rows": rows, "vocab": vocab, "temperature": temperature}


def _accept(name, seqs, nodes, children, vocab, drawn, temperature=1.0):
    """`children`: about how many a node has (1: chains).  `drawn`: the drafter drew its tokens from distributions that
    are handed over; otherwise it chose its most probable ones."""
    return {"name": name, "kind": "accept", "seqs": seqs, "nodes": nodes, "children": children, "vocab": vocab,
            "drawn": drawn, "temperature": temperature}


def listed():
    return [
        # decoding: one token per step of a batch of 64 slots, some of them idle
        _append("append 56 + 8 idle", seqs=56, lo=1, hi=1500, pad=8),
        # prompts of 16 sequences, 512 tokens each behind up to 90 earlier ones: the largest write
        _append("append 16 prompts", kv=32, page=16, seqs=16, new=512, lo=0, hi=90),
        # the verifier without a draft: 7B heads over image and instruction
        _attend("attend 281", kv=32, page=16, lo=281, hi=281),
        # the float32 reference model's kind of head, a batch with an empty slot
        _attend("attend f32 ragged", "f32", heads=16, kv=4, d=64, page=32, seqs=24, lo=0, hi=1500),
        # a long history for a single sequence: split over the length
        _attend("attend 131071", page=256, lo=131071, hi=131071),
        # many sequences served together
        _attend("attend 64 x 8192", seqs=64, lo=17, hi=8192),
        # streaming: the last 1024 tokens and four first ones, heads of 96 in groups of 7
        _attend("attend window 1024", heads=28, kv=4, d=96, page=32, seqs=48, lo=500, hi=20000, window=1024, sink=4),
        # the action tokens of a 60-node tree
        _probs("probs 60 actions", 60, ACTIONS, 0.7),
        # all tokens of 16 such trees
        _probs("probs 960 x 32000", 960, 32000),
        # the benchmark's tree over the action tokens, the drafter's most probable candidates
        _accept("accept tree of actions", 1, 60, 4, ACTIONS, False),
        # trees of drawn tokens, whole vocabulary
        _accept("accept 16 trees", 16, 60, 3, 32000, True),
        # chains of five drawn tokens, a large odd vocabulary
        _accept("accept 128 chains", 128, 6, 1, 128259, True, 0.9),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("append", "attend", "probs", "accept"), (3, 6, 2, 4))[0]
    if kind in ("append", "attend"):
        dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
        kv = rng.choice((1, 2, 4, 5, 8, 16, 32))
        heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16, 20, 64) if kv * g <= 128])
        d = rng.choice((64, 128, 128, 128, 40, 80, 96, 192, 256))
        page = rng.choice((16, 16, 32, 48, 64, 128, 256, 1024))
        row = 2 * kv * d * (2 if dtype == "bf16" else 4)            # bytes of a cached token
    if kind == "append":
        most = max(1, min(8000, 16 * 512 * 96 * 128 // ((heads + 2 * kv) * d)))       # tokens of a call
        tokens = _log_int(rng, 1, most)
        seqs = rng.randint(1, min(tokens, 64))
        page = page if row * seqs * page < 3e8 else 16
        c = _append("", dtype, heads, kv, d, page, seqs, tokens // seqs, 0, _log_int(rng, 1, max(1, min(100000, int(3e8) // (row * seqs)))),
                    rng.choice((0, 0, 1, 9)))
        c["lo"] = rng.randint(0, c["hi"])
        c["theta"] = rng.choice((1e4, 1e4, 5e5))
    elif kind == "attend":
        # (the largest listed one: 64 x 4104 tokens of 4096 bytes, for 32 heads of 128)
        keys = _log_int(rng, 40, min(int(1.05e9) // row, int(1.05e9) // (heads * d)))
        seqs = min(_log_int(rng, 1, 192), keys)
        page = page if row * seqs * page < 5e8 else 16
        hi = max(1, min(keys // seqs, 131072))
        c = _attend("", dtype, heads, kv, d, page, seqs, rng.randint(0, hi) if seqs > 1 else hi, hi)
        if rng.random() < 0.35:
            c["window"] = _log_int(rng, 1, max(1, hi))
            c["sink"] = rng.choice((0, 1, 4, 16, 33, 100))
    elif kind == "probs":
        vocab = rng.choice((_log_int(rng, 2, 160000), ACTIONS, 32000))
        c = _probs("", _log_int(rng, 1, max(1, min(2000, 30720000 // vocab))), vocab, rng.choice((1.0, 0.6, 0.8, 1.3)))
    else:
        children = rng.choice((1, 1, 2, 3, 5))
        vocab = rng.choice((_log_int(rng, 2, 130000), ACTIONS, 32000))
        nodes = rng.randint(1, 9) if children == 1 else rng.randint(2, 128)
        c = _accept("", _log_int(rng, 1, max(1, min(256, 98000000 // (vocab * nodes)))), nodes, children, vocab,
                    rng.random() < 0.6, rng.choice((1.0, 0.7, 1.4)))
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------------------

class _State:
    pass


def _spread(lo, hi, n, rng):
    """n whole numbers from lo to hi, evenly spread, in random order (so that their sum is known)."""
    v = np.rint(np.linspace(lo, hi, n)).astype(np.int64) if n > 1 else np.array([hi], dtype=np.int64)
    rng.shuffle(v)
    return v


def _lengths(case):
    return _spread(case["lo"], case["hi"], case["seqs"], np.random.default_rng(0))


def _table(lens, page, rng):
    """Pages of every sequence, scattered over a pool that has a few spare ones: block table (-1: none), pool size."""
    need = -(-lens // page)
    n_pages = int(need.sum()) + 3
    order = rng.permutation(n_pages)
    table = np.full((len(lens), max(1, int(need.max()))), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _pool(case, n_pages, gen):
    shape = (n_pages, case["kv"], case["page"], case["d"])
    out = []
    for _ in range(2):
        t = torch.empty(shape, dtype=_dtype(case), device=DEVICE)
        step = max(1, (1 << 26) // (t[0].numel()))
        for i in range(0, n_pages, step):
            part = t[i:i + step]
            part.copy_(torch.randn(part.shape, generator=gen, device=DEVICE))
        out.append(t)
    return out


def _prepare_append(case, seed, rng, gen):
    s = _State()
    before, new = _spread(case["lo"], case["hi"], case["seqs"], rng), case["new"]
    table, n_pages = _table(before + new, case["page"], rng)
    s.k_pool, s.v_pool = _pool(case, n_pages, gen)
    seq = np.repeat(np.arange(case["seqs"]), new)
    pos = (before[:, None] + np.arange(new)[None, :]).reshape(-1)
    seq, pos = np.concatenate([seq, np.full(case["pad"], -1)]), np.concatenate([pos, np.zeros(case["pad"], dtype=np.int64)])
    s.table = torch.from_numpy(table).to(DEVICE)
    s.seq = torch.from_numpy(seq.astype(np.int32)).to(DEVICE)
    s.pos = torch.from_numpy(pos.astype(np.int32)).to(DEVICE)
    n, hq, hk, d = len(seq), case["heads"], case["kv"], case["d"]
    # one row of a fused projection per token: queries, keys, values
    s.qkv = torch.randn(n, (hq + 2 * hk) * d, generator=gen, device=DEVICE)
    s.q = s.qkv[:, :hq * d].unflatten(1, (hq, d))
    s.k = s.qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
    s.v = s.qkv[:, (hq + hk) * d:].unflatten(1, (hk, d))
    s.q_out = torch.zeros(n, hq, d, device=DEVICE)
    s.status = torch.zeros(n, dtype=torch.int32, device=DEVICE)
    return s


def _prepare_attend(case, seed, rng, gen):
    s = _State()
    lens = _spread(case["lo"], case["hi"], case["seqs"], rng)
    table, n_pages = _table(lens, case["page"], rng)
    s.k_pool, s.v_pool = _pool(case, n_pages, gen)
    # rows behind the end of a sequence were never written
    for b in np.nonzero(lens % case["page"])[0]:
        last = table[b, lens[b] // case["page"]]
        s.k_pool[last, :, lens[b] % case["page"]:] = float("nan")
        s.v_pool[last, :, lens[b] % case["page"]:] = float("nan")
    s.table = torch.from_numpy(table).to(DEVICE)
    s.lens = torch.from_numpy(lens.astype(np.int32)).to(DEVICE)
    s.max_len = int(lens.max())
    # (a factor of two: scores that spread, as trained heads' do)
    s.q = 2.0 * torch.randn(case["seqs"], case["heads"], case["d"], generator=gen, device=DEVICE)
    s.out = torch.zeros_like(s.q)
    s.lse = torch.zeros(case["seqs"], case["heads"], device=DEVICE)
    s.status = torch.zeros(case["seqs"], dtype=torch.int32, device=DEVICE)
    return s


def _prepare_probs(case, seed, rng, gen):
    s = _State()
    s.logits = 3.0 * torch.randn(case["rows"], case["vocab"], generator=gen, device=DEVICE)
    s.probs = torch.empty_like(s.logits)
    return s


def _parents(case, rng):
    """Breadth first trees: a node's children follow those of the node before it."""
    T, kids, out = case["nodes"], case["children"], []
    for _ in range(case["seqs"]):
        parent, node = [-1], 0
        while len(parent) < T:
            for _ in range(1 if kids == 1 else int(rng.integers(1, 2 * kids))):
                if len(parent) < T:
                    parent.append(node)
            node += 1
        out.append(parent)
    return np.array(out, dtype=np.int32)


def _depth_cap(case):
    return 31 if case["children"] > 1 else max(1, case["nodes"] - 1)


def _prepare_accept(case, seed, rng, gen):
    s = _State()
    B, T, V = case["seqs"], case["nodes"], case["vocab"]
    parent = _parents(case, rng)
    z = 3.0 * torch.randn(B * T, V, generator=gen, device=DEVICE)
    s.target = torch.softmax(z / case["temperature"], dim=1)
    # the drafter's idea of it
    z.add_(torch.randn(B * T, V, generator=gen, device=DEVICE))
    s.draft = torch.softmax(z / case["temperature"], dim=1)
    lo = 32000 - ACTIONS if V == ACTIONS else 0
    s.lo = lo
    token = torch.full((B, T), lo, dtype=torch.int32, device=DEVICE)
    draft = s.draft.view(B, T, V)
    if case["drawn"]:
        up = torch.from_numpy(np.maximum(parent, 0).astype(np.int64)).to(DEVICE)
        for c in range(1, T):
            row = draft[torch.arange(B, device=DEVICE), up[:, c]]
            noise = torch.empty_like(row).exponential_(generator=gen)
            token[:, c] = lo + (row / noise).argmax(1).to(torch.int32)
    else:
        up = np.maximum(parent, 0)
        rank = np.zeros((B, T), dtype=np.int64)                        # which child of its parent a node is
        for c in range(2, T):
            rank[:, c] = np.where(parent[:, c] == parent[:, c - 1], rank[:, c - 1] + 1, 0)
        best = draft.topk(min(int(rank.max()) + 1, V), dim=2).indices
        at = [torch.from_numpy(t).to(DEVICE) for t in (up.astype(np.int64), np.minimum(rank, V - 1))]
        token[:, 1:] = (lo + best[torch.arange(B, device=DEVICE)[:, None], at[0], at[1]])[:, 1:].to(torch.int32)
    s.token = token.reshape(-1)
    if not case["drawn"]:
        s.draft = None
    s.u_accept = torch.rand(B * T, generator=gen, device=DEVICE)
    s.u_draw = torch.rand(B, generator=gen, device=DEVICE)
    s.parent_host = parent
    s.parent = torch.from_numpy(parent).to(DEVICE)
    s.d_cap = _depth_cap(case)
    s.accept_mask = torch.zeros(B * T, dtype=torch.uint8, device=DEVICE)
    s.accepted_len, s.best_node, s.status = (torch.zeros(B, dtype=torch.int32, device=DEVICE) for _ in range(3))
    s.path, s.out_tokens = (torch.zeros(B, s.d_cap + 1, dtype=torch.int32, device=DEVICE) for _ in range(2))
    return s


_PREPARE = {"append": _prepare_append, "attend": _prepare_attend, "probs": _prepare_probs, "accept": _prepare_accept}


def _inputs(case, seed):
    rng = np.random.default_rng([seed, 17])
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    return _PREPARE[case["kind"]](case, seed, rng, gen)


def prepare(case, seed):
    s = _inputs(case, seed)
    s.case = case
    if own:
        from paper_2507_22424_amd import binding as sv
        s.sv = sv
        if case["kind"] in ("append", "attend"):
            s.cache = sv.PagedCache(s.k_pool, s.v_pool, s.table)
        if case["kind"] == "attend":
            s.workspace = torch.empty(sv.sv_paged_workspace_bytes(s.cache, case["heads"], s.max_len), dtype=torch.uint8, device=DEVICE)
        if case["kind"] == "accept":
            s.tree = sv.DeviceTree(s.parent_host, case["seqs"], case["nodes"], s.d_cap, DEVICE)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------

def _plain_append(s, c):
    seq, pos = s.seq.long(), s.pos.long()
    ok = seq >= 0
    half = c["d"] // 2
    inv = c["theta"] ** (-2.0 * torch.arange(half, dtype=torch.float64, device=DEVICE) / c["d"])
    angle = pos.double()[:, None] * inv[None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def rotate(x, n=len(seq)):
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos[:n] - b * sin[:n], b * cos[:n] + a * sin[:n]], dim=-1)

    s.q_out.copy_(torch.where(ok[:, None, None], rotate(s.q), s.q_out))
    page = s.table[seq.clamp(min=0), pos // c["page"]].long()
    n = c["seqs"] * c["new"]                                          # padding comes behind
    page, row = page[:n], (pos % c["page"])[:n]
    s.k_pool[page, :, row] = rotate(s.k[:n], n).to(s.k_pool.dtype)
    s.v_pool[page, :, row] = s.v[:n].to(s.v_pool.dtype)
    s.status.copy_((~ok).int())
    return s.q_out, s.k_pool, s.v_pool, s.status


def _plain_attend(s, c):
    B, H, G, d, page = c["seqs"], c["kv"], c["heads"] // c["kv"], c["d"], c["page"]
    lens = s.lens.long()
    if c["window"]:
        sink, window = min(c["sink"], s.max_len), min(c["window"], s.max_len)
        first = (lens - window).clamp(min=0)[:, None]
        idx = torch.cat([torch.arange(sink, device=DEVICE).expand(B, sink), first + torch.arange(window, device=DEVICE)], 1)
        seen = idx < lens[:, None]
        seen[:, sink:] &= idx[:, sink:] >= sink                       # (counted among the first ones already)
    else:
        idx = torch.arange(s.max_len, device=DEVICE).expand(B, s.max_len)
        seen = idx < lens[:, None]
    at = torch.where(seen, idx, 0)
    rows = s.table.long().gather(1, at // page).clamp(min=0) * page + at % page
    out, lse = torch.empty_like(s.out), torch.empty_like(s.lse)
    step = max(1, (1 << 28) // max(1, idx.shape[1] * H * d))           # sequences at once
    for b in range(0, B, step):
        r, ok = rows[b:b + step], seen[b:b + step]
        k = s.k_pool.transpose(1, 2)[r // page, r % page].float().transpose(1, 2).masked_fill_(~ok[:, None, :, None], 0.0)
        q = s.q[b:b + step].view(-1, H, G, d)
        score = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
        del k
        score.masked_fill_(~ok[:, None, None, :], float("-inf"))
        top = score.amax(-1, keepdim=True).clamp(min=-1e30)
        e = torch.exp(score - top)
        total = e.sum(-1, keepdim=True)
        v = s.v_pool.transpose(1, 2)[r // page, r % page].float().transpose(1, 2).masked_fill_(~ok[:, None, :, None], 0.0)
        o = torch.matmul(e, v.contiguous()) / torch.where(total > 0, total, 1.0)
        out[b:b + step] = o.reshape(-1, c["heads"], d)
        lse[b:b + step] = torch.where(total > 0, top + torch.log(total), float("-inf")).reshape(-1, c["heads"])
    return out, lse, s.status


def _plain_probs(s, c):
    z = s.logits / c["temperature"]
    e = torch.exp(z - z.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_accept(s, c):
    """All sequences side by side, node after node: a node's children have higher numbers than it has."""
    B, T, V, lo = c["seqs"], c["nodes"], c["vocab"], s.lo
    b = torch.arange(B, device=DEVICE)
    p_all = s.target.view(B, T, V)
    q_all = s.draft.view(B, T, V) if s.draft is not None else None
    token, u = s.token.view(B, T), s.u_accept.view(B, T).double()
    cur = torch.zeros(B, dtype=torch.int64, device=DEVICE)
    depth = torch.zeros_like(cur)
    less, mass = torch.zeros(B, dtype=torch.float64, device=DEVICE), torch.ones(B, dtype=torch.float64, device=DEVICE)
    mask = torch.zeros(B, T, dtype=torch.uint8, device=DEVICE)
    mask[:, 0] = 1
    path = torch.full((B, s.d_cap + 1), -1, dtype=torch.int32, device=DEVICE)
    path[:, 0] = 0
    tokens = torch.full_like(path, -1)
    refused = torch.zeros(B, V, dtype=torch.bool, device=DEVICE)
    for n in range(1, T):
        tried = (s.parent[:, n] == cur) & (depth < s.d_cap)
        x = token[:, n].long() - lo
        inside = (x >= 0) & (x < V)
        x = x.clamp(0, V - 1)
        p = torch.where(inside, p_all[b, cur, x].double(), 0.0)
        if q_all is not None:
            q = torch.where(inside, q_all[b, cur, x].double(), 0.0)
            take = tried & (u[:, n] * q * mass < (p - less * q).clamp(min=0.0))
            drop = tried & ~take
            less = torch.where(drop, less + mass, less)
            rest = (p_all[b, cur].double() - less[:, None] * q_all[b, cur].double()).clamp_(min=0.0).sum(1)
            mass = torch.where(drop, rest, mass)
        else:
            p = torch.where(refused[b, x], 0.0, p)
            take = tried & (u[:, n] * mass < p)
            drop = tried & ~take
            mass = torch.where(drop, (mass - p).clamp(min=0.0), mass)
            refused[b, x] |= drop & inside
        depth = depth + take
        cur = torch.where(take, n, cur)
        less, mass = torch.where(take, 0.0, less), torch.where(take, 1.0, mass)
        refused &= ~take[:, None]
        mask[:, n] = take
        path[b, depth] = torch.where(take, n, path[b, depth])
        up = (depth - 1).clamp(min=0)
        tokens[b, up] = torch.where(take, token[:, n], tokens[b, up])
    p = p_all[b, cur].double()
    left = (p - less[:, None] * q_all[b, cur].double()).clamp_(min=0.0) if q_all is not None else p.masked_fill(refused, 0.0)
    none = ~(left.sum(1) > 0)
    left = torch.where(none[:, None], p, left)
    cum = torch.cumsum(left, 1)
    at = (cum <= s.u_draw.double()[:, None] * left.sum(1, keepdim=True)).sum(1)
    last = torch.where(left > 0, torch.arange(V, device=DEVICE), 0).amax(1)
    tokens[b, depth] = (lo + torch.minimum(at, last)).to(torch.int32)
    return mask.view(-1), depth.to(torch.int32), cur.to(torch.int32), path, tokens, none.to(torch.int32)


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "probs": _plain_probs, "accept": _plain_accept}


# ---- the framework's calls ---------------------------------------------------------------------------------

def _own_append(s, c):
    s.sv.sv_paged_append(s.cache, s.seq, s.pos, s.q, s.k, s.v, s.q_out, c["theta"], s.status)
    return s.q_out, s.k_pool, s.v_pool, s.status


def _own_attend(s, c):
    s.sv.sv_paged_attention(s.cache, s.lens, s.max_len, s.q, 1.0 / math.sqrt(c["d"]), c["window"], c["sink"], s.out,
                            s.lse, s.status, s.workspace)
    return s.out, s.lse, s.status


def _own_probs(s, c):
    s.sv.sv_token_probs(s.logits, c["temperature"], s.probs)
    return s.probs


def _own_accept(s, c):
    s.sv.sv_sampled_accept(s.tree.struct, s.token, s.target, s.draft, s.lo, s.u_accept, s.u_draw, c["seqs"], s.d_cap,
                           s.accept_mask, s.accepted_len, s.best_node, s.path, s.out_tokens, s.status)
    return s.accept_mask, s.accepted_len, s.best_node, s.path, s.out_tokens, s.status


_OWN = {"append": _own_append, "attend": _own_attend, "probs": _own_probs, "accept": _own_accept}


def run(state):
    return (_OWN if own else _PLAIN)[state.case["kind"]](state, state.case)


# ---- what a pass cannot do without -------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("append", "attend"):
        e, hq, hk, d = 4 if case["dtype"] == "f32" else 2, case["heads"], case["kv"], case["d"]
    if kind == "append":
        n = case["seqs"] * case["new"]
        return {"bytes": n * (8 * hq * d + 2 * (4 + e) * hk * d), "flops": n * 3 * (hq + hk) * d}
    if kind == "attend":
        seen = [min(int(l), case["sink"]) + min(max(0, int(l) - case["sink"]), case["window"]) if case["window"] else int(l)
                for l in _lengths(case)]
        return {"bytes": sum(seen) * 2 * e * hk * d + 8 * case["seqs"] * hq * d, "flops": 4 * sum(seen) * hq * d}
    if kind == "probs":
        n = case["rows"] * case["vocab"]
        return {"bytes": 8 * n, "flops": 4 * n}
    n = case["seqs"] * case["vocab"]
    return {"bytes": (8 if case["drawn"] else 4) * n + 16 * case["seqs"] * case["nodes"], "flops": 4 * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def _exact_append(s, c):
    seq, pos, table = s.seq.tolist(), s.pos.tolist(), s.table.tolist()
    q, k, v = s.q.double(), s.k.double(), s.v.double()
    i = torch.arange(c["d"] // 2, dtype=torch.float64, device=DEVICE)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       s.pos.double()[:, None] * torch.exp(i * (-2.0 * math.log(c["theta"]) / c["d"])))[:, None, :]

    def turned(x):
        z = torch.complex(*x.chunk(2, dim=-1)) * turn
        return torch.cat([z.real, z.imag], -1)

    rq, rk = turned(q), turned(k)
    kp, vp = s.k_pool.double(), s.v_pool.double()
    real = [t for t in range(len(seq)) if seq[t] >= 0]
    slot = torch.tensor([table[seq[t]][pos[t] // c["page"]] * c["page"] + pos[t] % c["page"] for t in real], device=DEVICE)
    t = torch.tensor(real, device=DEVICE)
    for pool, new in ((kp, rk), (vp, v)):
        flat = pool.permute(0, 2, 1, 3).reshape(-1, c["kv"], c["d"]).index_copy(0, slot, new[t])
        pool.copy_(flat.view(pool.shape[0], c["page"], c["kv"], c["d"]).permute(0, 2, 1, 3))
    q_out = torch.zeros_like(rq)
    q_out[t] = rq[t]
    return q_out, kp, vp, torch.tensor([int(x < 0) for x in seq], dtype=torch.int32, device=DEVICE)


def _exact_attend(s, c):
    out, lse = s.out.double(), s.lse.double()
    G, page = c["heads"] // c["kv"], c["page"]
    for b, n in enumerate(s.lens.tolist()):
        first = max(0, n - c["window"]) if c["window"] else 0
        keys = sorted(set(range(min(n, c["sink"] if c["window"] else 0))) | set(range(first, n)))
        if not keys:
            out[b], lse[b] = 0.0, float("-inf")
            continue
        j = torch.tensor(keys, device=DEVICE)
        g = s.table[b].long()[j // page]
        for h in range(c["kv"]):
            k, v = s.k_pool[g, h, j % page].double(), s.v_pool[g, h, j % page].double()
            x = (s.q[b, h * G:(h + 1) * G].double()[:, None, :] * k[None]).sum(-1) / math.sqrt(c["d"]) if G * len(keys) * c["d"] < 1 << 24 \
                else s.q[b, h * G:(h + 1) * G].double() @ k.T.contiguous() / math.sqrt(c["d"])
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(x, 1)
            out[b, h * G:(h + 1) * G] = torch.exp(x - lse[b, h * G:(h + 1) * G, None]) @ v
    return out, lse, torch.zeros_like(s.status)


def _exact_probs(s, c):
    return torch.stack([torch.exp(torch.log_softmax(r.double() / c["temperature"], 0)) for r in s.logits])


def _exact_accept(s, c):
    """One sequence after the other, the residual distribution itself carried along."""
    B, T, V = c["seqs"], c["nodes"], c["vocab"]
    token, u, parent = s.token.view(B, T).cpu().numpy(), s.u_accept.view(B, T).cpu().numpy().astype(float), s.parent_host
    u_draw = s.u_draw.cpu().numpy().astype(float)
    mask = np.zeros((B, T), dtype=np.uint8)
    length, best, status = (np.zeros(B, dtype=np.int32) for _ in range(3))
    path, out = (np.full((B, s.d_cap + 1), -1, dtype=np.int32) for _ in range(2))
    for b in range(B):
        node, walk = 0, [0]
        while True:
            p = s.target[b * T + node].cpu().numpy().astype(float)
            now, q, gone = p.copy(), None, 1.0
            if s.draft is not None:
                q = s.draft[b * T + node].cpu().numpy().astype(float)
            down = None
            for child in np.nonzero(parent[b] == node)[0] if len(walk) <= s.d_cap else ():
                x = int(token[b, child]) - s.lo
                px = now[x] if 0 <= x < V else 0.0
                if q is not None:
                    if u[b, child] * (q[x] if 0 <= x < V else 0.0) < px:
                        down = int(child)
                        break
                    now = np.maximum(now - q, 0.0)
                    if now.sum() > 0:
                        now /= now.sum()
                else:
                    if u[b, child] * gone < px:
                        down = int(child)
                        break
                    gone = max(gone - px, 0.0)
                    if 0 <= x < V:
                        now[x] = 0.0
            if down is None:
                break
            out[b, len(walk) - 1] = token[b, down]
            walk.append(down)
            node = down
        if not now.sum() > 0:
            status[b], now = 1, p
        cum = np.cumsum(now)
        at = int(np.searchsorted(cum, u_draw[b] * cum[-1], side="right"))
        out[b, len(walk) - 1] = s.lo + min(at, int(np.nonzero(now)[0][-1]))
        mask[b, walk] = 1
        path[b, :len(walk)] = walk
        length[b], best[b] = len(walk) - 1, node
    return tuple(torch.from_numpy(t).to(DEVICE) for t in (mask.reshape(-1), length, best, path, out, status))


_EXACT = {"append": _exact_append, "attend": _exact_attend, "probs": _exact_probs, "accept": _exact_accept}


def exact(case, seed):
    return _EXACT[case["kind"]](_inputs(case, seed), case)
