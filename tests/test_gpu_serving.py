"""The calls around the tree pass on an MI355X: sampled acceptance and probabilities, paged cache with append and
attention of one new token - against float64, at the sizes and masks where they can go wrong.

Tolerances count roundings, u = 2^-24 (half a step of float32 at 1), worst case over the order of the sums:
  scores     products and sums of d terms: (d + 8) u of sum |q k| scale, queries and scale rounded among them
  weights    twice that (score and maximum) + 8 u (exponential, log2 e, split)
  outputs    weights' error + one u per term of the longest chain of sums, of the largest |V|
"""
import numpy as np
import pytest
import torch

from oracle import paged_cache as pc
from oracle import sampled_accept as sa
from paper_2507_22424_amd import binding as sv
from paper_2507_22424_amd import workload as wl
from paper_2507_22424_amd.runner import VerifyPass

from parity_utils import f64, say

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- probabilities ------------------------------------------------------------------------------

def _softmax(z, t):
    z = z / t
    with np.errstate(invalid="ignore"):
        top = z.max(1, keepdims=True)
        e = np.exp(z - np.where(np.isneginf(top), 0.0, top))
        return np.where(np.isneginf(top), 0.0, e / np.where(e.sum(1, keepdims=True) == 0, 1.0, e.sum(1, keepdims=True)))


def _check_probs(got, z, t):
    want = _softmax(z, t)
    nan = np.isnan(z).any(1) | np.isposinf(z).any(1)
    assert np.isnan(got[nan]).all()
    got, want, z = got[~nan], want[~nan], z[~nan]
    # exponent x = (z - max) / t: difference and two factors round, 3u |x|; exponential, quotient, sum of n terms
    top = np.where(np.isneginf(z.max(1, keepdims=True)), 0.0, z.max(1, keepdims=True))
    x = np.minimum(np.where(np.isneginf(z), 0.0, (top - z) / t), 100.0)
    tol = want * (3 * U * (x + (x * want).sum(1, keepdims=True)) + (z.shape[1] / 64 + 24) * U) + 1e-37
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("rows,n", [(1, 1), (3, 2), (60, 256), (7, 255), (5, 257), (2, 2047), (3, 2048), (3, 2049), (9, 4099), (4, 32000),
                                    (2, 32001), (1, 65539), (3, 128259), (1, 300001), (2100, 33)])
def test_token_probs(rows, n):
    gen = torch.Generator().manual_seed(rows * 7 + n)
    for t, size in ((1.0, 3.0), (0.7, 30.0), (1e-3, 1.0), (50.0, 1000.0)):
        z = size * torch.randn(rows, n, generator=gen)
        if rows > 2:
            z[0] = -float("inf")                     # nothing left
            z[1, 1:] = -float("inf")                 # one token left
            z[2, ::2] = torch.finfo(torch.float32).min
        if rows > 4:
            z[3, n // 2] = float("nan")
            z[4, n - 1] = float("inf")
        d = z.cuda()
        p = torch.full((rows, n), -1.0, device="cuda")
        sv.sv_token_probs(d, t, p)
        assert torch.equal(d.cpu().nan_to_num(7.0), z.nan_to_num(7.0))
        t32 = float(np.float32(t))
        _check_probs(f64(p.cpu()), f64(z), t32)
        sv.sv_token_probs(d, t, d)                   # in place
        assert torch.equal(d.nan_to_num(7.0), p.nan_to_num(7.0))


def test_token_probs_at_unaligned_rows():
    """Rows of odd length begin at every alignment, and so may the tensors."""
    z = 4 * torch.randn(5, 1003, generator=torch.Generator().manual_seed(3))
    for off in range(4):
        buf = torch.full((5 * 1003 + 8,), 9.0, device="cuda")
        src = torch.zeros(5 * 1003 + 8, device="cuda")
        src[off:off + 5 * 1003] = z.reshape(-1).cuda()
        for to in range(4):
            out = buf.clone()
            sv.sv_token_probs(src[off:off + 5 * 1003].view(5, 1003), 1.0, out[to:to + 5 * 1003].view(5, 1003))
            _check_probs(f64(out[to:to + 5 * 1003].view(5, 1003).cpu()), f64(z), 1.0)
            assert (out[:to] == 9).all() and (out[to + 5 * 1003:] == 9).all()


# ---- sampled acceptance ---------------------------------------------------------------------------

class Accept:
    """Device buffers of sv_sampled_accept for B trees of T nodes."""

    def __init__(self, parents, d_cap):
        self.B, self.T, self.d_cap = len(parents), len(parents[0]), d_cap
        self.parents = np.asarray(parents, dtype=np.int32)
        self.parent = torch.from_numpy(self.parents).cuda()
        self.tree = sv.Tree(self.parent.data_ptr(), None, None, self.T, (self.T + 63) // 64)
        self.mask = torch.zeros(self.B * self.T, dtype=torch.uint8, device="cuda")
        self.length, self.best, self.status = (torch.zeros(self.B, dtype=torch.int32, device="cuda") for _ in range(3))
        self.path, self.tokens = (torch.zeros(self.B, d_cap + 1, dtype=torch.int32, device="cuda") for _ in range(2))

    def outputs(self):
        return (self.mask, self.length, self.best, self.path, self.tokens, self.status)

    def call(self, tok, p, q, lo, u, ud):
        for t in self.outputs():
            t.fill_(99)
        sv.sv_sampled_accept(self.tree, tok, p, q, lo, u, ud, self.B, self.d_cap, *self.outputs())

    def check(self, tok, p, q, lo, u, ud):
        """tok [B, T], p, q [B, T, V], u [B, T], ud [B]: numpy; against the oracle."""
        dev = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()
        self.call(dev(tok.reshape(-1), torch.int32), dev(p.reshape(self.B * self.T, -1), torch.float32),
                  None if q is None else dev(q.reshape(self.B * self.T, -1), torch.float32), lo, dev(u.reshape(-1), torch.float32),
                  dev(ud, torch.float32))
        got = [t.cpu().numpy() for t in self.outputs()]
        f = lambda a: np.asarray(a, dtype=np.float32).astype(np.float64)
        for b in range(self.B):
            want = sa.sampled_accept(self.parents[b], tok[b], f(p[b]), None if q is None else f(q[b]), lo, f(u[b]), float(f(ud[b])),
                                     self.d_cap)
            n = want["length"]
            assert int(got[1][b]) == n and int(got[2][b]) == want["best"] and int(got[5][b]) == want["status"], b
            assert got[0].reshape(self.B, self.T)[b].astype(bool).tolist() == want["mask"].tolist(), b
            assert got[3][b].tolist() == want["path"] + [-1] * (self.d_cap - n), b
            assert got[4][b].tolist() == want["tokens"] + [-1] * (self.d_cap - n), b
        return got


def _trees(B, T, dmax, kids, rng):
    return [wl.draft_tree(T, dmax, kids, min(dmax, T - 1), rng) for _ in range(B)]


def _draft_tokens(parents, q, rng, drawn):
    """Tokens drawn from the parent's row of q [B, T, V], or its most probable ones in turn."""
    B, T, V = q.shape
    tok = np.zeros((B, T), dtype=np.int64)
    for b in range(B):
        seen = {}
        for c in range(1, T):
            row = q[b, parents[b][c]]
            if drawn:
                tok[b, c] = min(int(np.searchsorted(np.cumsum(row), rng.random() * row.sum(), side="right")), V - 1)
            else:
                k = seen.get(parents[b][c], 0)
                seen[parents[b][c]] = k + 1
                tok[b, c] = np.argsort(-row, kind="stable")[min(k, V - 1)]
    return tok


def _probs(rng, shape, spread):
    z = spread * rng.standard_normal(shape)
    e = np.exp(z - z.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("B,T,dmax,kids,V", [(1, 1, 7, 3, 5), (2, 2, 7, 1, 1), (9, 7, 6, 1, 256), (5, 15, 7, 3, 2), (6, 60, 7, 4, 256),
                                             (3, 64, 7, 6, 257), (3, 65, 9, 5, 1023), (2, 128, 7, 6, 2049), (2, 26, 5, 4, 32000),
                                             (2, 9, 8, 1, 70001), (1, 12, 4, 4, 200003), (40, 33, 31, 2, 40)])
def test_sampled_accept_equals_the_oracle(B, T, dmax, kids, V, drawn):
    rng = np.random.default_rng(B * 1000 + T * 10 + V)
    a = Accept(_trees(B, T, dmax, kids, rng), dmax)
    lengths = []
    for trial in range(3):
        p = _probs(rng, (B, T, V), [1.0, 2.5, 0.1][trial])
        q = _probs(rng, (B, T, V), 1.0) if trial == 1 else _probs(rng, (B, T, V), 0.3) * 0.2 + p * np.float32(0.8)
        tok = _draft_tokens(a.parents, q.astype(np.float64), rng, drawn) + 31
        if trial == 2 and T > 4:
            tok[:, 2] = 5                            # below the columns
            tok[:, 3] = 31 + V                       # above
            tok[:, 4] = -2 ** 31
        got = a.check(tok, p, q if drawn else None, 31, rng.random((B, T)).astype(np.float32), rng.random(B).astype(np.float32))
        lengths += got[1].tolist()
    say(f"[sampled accept B={B} T={T} V={V} drawn={drawn}] accepted lengths {lengths}")


@pytest.mark.parametrize("drawn", [True, False])
def test_sampled_accept_corners(drawn):
    """Rows without mass, NaN, equal distributions, equal siblings, random numbers at the ends, a depth cap, and
    parents that are none."""
    rng = np.random.default_rng(5)
    B, T, V = 12, 10, 37
    parents = [[-1, 0, 0, 0, 1, 1, 2, 4, 4, 7]] * B
    p = _probs(rng, (B, T, V), 1.0)
    q = p.copy() if drawn else None
    tok = _draft_tokens(np.array(parents), p.astype(np.float64), rng, True)
    u, ud = rng.random((B, T)).astype(np.float32), rng.random(B).astype(np.float32)
    u[1], ud[1] = 0.0, 0.0
    u[2], ud[2] = 1 - 2.0 ** -24, 1 - 2.0 ** -24
    p[3] = 0.0                                       # no mass at all: the first token, status 3
    p[4, 0] = np.nan
    p[5, 0, ::2] = np.nan
    p[6, 0] = 0.0
    p[6, 0, 5] = 1.0                                 # one token only
    tok[6, 1:4] = 5
    u[6] = 0.999
    tok[7, 1:4] = tok[7, 1]                          # equal siblings
    u[7] = 0.9999
    if drawn:
        q[8] = 0.0                                   # tokens that q says cannot have been drawn
        q[9, 0] = p[9, 0] * 4                        # q above p everywhere: nothing is left after a refusal
        u[9] = 0.9999
        q[10, 0] = np.nan
    else:
        p[8, 0] = 0.0
        p[8, 0, tok[8, 1:4]] = np.float32(1e-3)      # all mass in the candidates: nothing is left
        u[8] = 0.9999
    ud[11], u[11] = np.nan, 1.0                      # no random numbers: nothing accepted, the last token
    for lo in (100, 0):                              # all tokens outside the columns, all inside
        for cap in (5, 2, 1, 0):
            a = Accept(parents, cap)
            got = a.check(tok, p, q, lo, u, ud)
            if cap == 5 and lo == 0:
                assert got[5][3] == 3 and got[5].tolist().count(1) >= 1
        bad = Accept([[5, 0, 7, -3, 1, 5, 2 ** 31 - 1, 6, 4, -1]] * B, 5)
        bad.check(tok, p, q, lo, u, ud)


def test_sampled_accept_on_exact_fractions():
    """Equal probabilities and random numbers that fall on the borders: 'exceeds' is strict on both sides."""
    V, T, B = 64, 5, 65
    p = np.full((B, T, V), 1.0 / V, dtype=np.float32)
    tok = np.tile(np.arange(T), (B, 1))
    u = np.full((B, T), 0.5, dtype=np.float32)
    ud = (np.arange(B) / np.float32(B - 1)).astype(np.float32)
    for q in (None, np.full((B, T, V), 2.0 / V, dtype=np.float32)):
        a = Accept([[-1, 0, 0, 0, 0]] * B, 4)
        a.check(tok, p, q, 0, u, ud)


def test_sampled_accept_reads_only_rows_of_the_walk_and_is_reproducible():
    rng = np.random.default_rng(8)
    B, T, V = 4, 20, 5000
    a = Accept(_trees(B, T, 5, 3, rng), 5)
    dev = lambda x, dt: torch.from_numpy(x).to(dt).cuda()
    p, q = _probs(rng, (B, T, V), 1.0), _probs(rng, (B, T, V), 1.0)
    args = (dev(_draft_tokens(a.parents, q.astype(float), rng, True).reshape(-1), torch.int32), dev(p.reshape(B * T, V), torch.float32),
            dev(q.reshape(B * T, V), torch.float32), 0, dev(rng.random(B * T).astype(np.float32), torch.float32),
            dev(rng.random(B).astype(np.float32), torch.float32))
    a.call(*args)
    want = [t.clone() for t in a.outputs()]
    keep = [t.clone() for t in args if torch.is_tensor(t)]
    for _ in range(3):
        a.call(*args)
        assert all(torch.equal(x, y) for x, y in zip(want, a.outputs()))
    assert all(torch.equal(x, y) for x, y in zip(keep, [t for t in args if torch.is_tensor(t)]))


@pytest.mark.parametrize("V", [256, 257, 1024, 1025, 4096, 4097, 16384, 16385, 32768, 32769])
def test_sampled_accept_of_many_refused_siblings(V):
    """Several sums over one row, at every node of the walk: random numbers near 1 refuse nearly all but the last of a
    node's children.  Lengths at which more threads take a row, and one that none hold."""
    rng = np.random.default_rng(V)
    parents = [[-1, 0, 0, 0, 0, 4, 4, 4, 7, 7, 7, 7], [-1, 0, 0, 0, 0, 0, 0, 1, 1, 6, 6, 6]]
    B, T = 2, 12
    a = Accept(parents, 6)
    for trial in range(3):
        p, q = _probs(rng, (B, T, V), 1.0), _probs(rng, (B, T, V), 1.0)
        tok = _draft_tokens(parents, q.astype(np.float64), rng, True)
        u = np.full((B, T), 0.999, dtype=np.float32)
        if trial:                                    # and the walk goes on behind a node's last child
            u[0, [4, 7]] = 0.0
            u[1, [6, 11]] = 0.0
        if trial == 2:
            p[0, 0, V // 2:] = np.nan                # has no mass
            q[:, 7, ::3] = np.nan
        a.check(tok, np.nan_to_num(p, nan=0.0), np.nan_to_num(q, nan=0.0), 0, u, rng.random(B).astype(np.float32))
        dev = lambda x, dt: torch.from_numpy(x).to(dt).cuda()
        want = [t.clone() for t in a.outputs()]
        ud = torch.tensor([0.25, 0.75], device="cuda")
        outs = []
        for pp, qq in ((p, q), (np.nan_to_num(p, nan=0.0), np.nan_to_num(q, nan=0.0))):
            a.call(dev(tok.reshape(-1), torch.int32), dev(pp.reshape(B * T, V), torch.float32), dev(qq.reshape(B * T, V), torch.float32), 0,
                   dev(u.reshape(-1), torch.float32), ud)
            outs.append([t.clone() for t in a.outputs()])
        assert all(torch.equal(x, y) for x, y in zip(*outs))
        assert torch.equal(want[0], outs[0][0])      # what is accepted does not hang on the draw


def test_sampled_accept_of_many_trees_is_that_of_few():
    """600 trees over rows that the workgroups of few trees hold."""
    rng = np.random.default_rng(3)
    few, n, T, V = 8, 600, 5, 16500
    p, q = _probs(rng, (few, T, V), 1.0), _probs(rng, (few, T, V), 1.0)
    u, ud = rng.random((few, T)).astype(np.float32), rng.random(few).astype(np.float32)
    parents = [[-1, 0, 0, 0, 3]] * few
    tok = _draft_tokens(parents, q.astype(np.float64), rng, True)
    a = Accept(parents, 3)
    a.check(tok, p, q, 0, u, ud)
    many = Accept([parents[0]] * n, 3)
    at = torch.arange(n, device="cuda") % few
    dev = lambda x, dt: torch.from_numpy(x).to(dt).cuda()[at]
    many.call(dev(tok, torch.int32).reshape(-1), dev(p, torch.float32).view(n * T, V), dev(q, torch.float32).view(n * T, V), 0,
              dev(u, torch.float32).reshape(-1), dev(ud, torch.float32))
    for x, y in zip(many.outputs(), a.outputs()):
        assert torch.equal(x.view(n, -1), y.view(few, -1)[at])


# ---- append ---------------------------------------------------------------------------------------

def _append_case(dtype, nq, nkv, d, page, max_pages, seqs, pos, theta=1e4, table=None, n_seqs=None, fused=True, with_q=True, in_place=False):
    rng = np.random.default_rng(len(pos) * 31 + d)
    gen = torch.Generator().manual_seed(d + page)
    n, S = len(pos), n_seqs or max(max(seqs) + 1, 1)
    n_pages = S * max_pages + 2
    if table is None:
        table = rng.permutation(n_pages)[:S * max_pages].reshape(S, max_pages).astype(np.int32)
    pool = [torch.randn(n_pages, nkv, page, d, generator=gen).to(DT[dtype]).cuda() for _ in range(2)]
    before = [t.clone() for t in pool]
    cache = sv.PagedCache(pool[0], pool[1], torch.from_numpy(table).cuda())
    width = (nq + 2 * nkv) * d
    qkv = torch.randn(n, width + (8 if fused else 0), generator=gen)
    dev = qkv.cuda()
    cut = lambda a, b: dev[:, a * d:b * d].unflatten(1, (b - a, d)) if fused else dev[:, a * d:b * d].unflatten(1, (b - a, d)).contiguous()
    q, k, v = cut(0, nq), cut(nq, nq + nkv), cut(nq + nkv, nq + 2 * nkv)
    q_out = q if in_place else torch.full((n, nq, d), 5.0, device="cuda")
    status = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    sv.sv_paged_append(cache, torch.tensor(seqs, dtype=torch.int32, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda"),
                       q if with_q else None, k, v, q_out if with_q else None, theta, status)
    got_k, got_v = f64(pool[0].cpu()), f64(pool[1].cpu())
    want_k, want_v = f64(before[0].cpu()), f64(before[1].cpu())
    x = f64(qkv)
    th = float(np.float32(theta))
    tol_k = np.zeros_like(want_k)
    half_step = 2.0 ** -8 if dtype == "bf16" else U
    want_status = []
    for t in range(n):
        s, p = seqs[t], pos[t]
        st = 1 if s < 0 else 2 if s >= S or p < 0 or p // page >= max_pages else 4 if not 0 <= table[s, p // page] < n_pages else 0
        want_status.append(st)
        qt = x[t, :nq * d].reshape(nq, d)
        if with_q and not in_place:
            if st:
                assert (q_out[t] == 5).all()
            else:
                # angle in turns: rounded to float32 once (2^-25 of half a turn: 0.8 u), sine and cosine 2 u each, products
                # and sum: below 8 u of |x| + |y|
                tol = 8 * U * (np.abs(qt) + np.abs(np.roll(qt, d // 2, axis=-1)))
                assert (np.abs(f64(q_out[t].cpu()) - pc.rotate(qt, p, th)) <= tol).all(), t
        if st:
            continue
        g, r = table[s, p // page], p % page
        kt = x[t, nq * d:(nq + nkv) * d].reshape(nkv, d)
        want_k[g, :, r] = pc.rotate(kt, p, th)
        tol_k[g, :, r] = 8 * U * (np.abs(kt) + np.abs(np.roll(kt, d // 2, axis=-1))) * (1 + half_step) + half_step * np.abs(want_k[g, :, r])
        want_v[g, :, r] = f64(qkv[t, (nq + nkv) * d:(nq + 2 * nkv) * d].reshape(nkv, d).to(DT[dtype]))
    assert status.cpu().tolist() == want_status
    assert (np.abs(got_k - want_k) <= tol_k).all()          # (rows that no token went to: bit for bit)
    assert np.array_equal(got_v, want_v)
    return q_out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,d,page", [(32, 8, 128, 64), (4, 4, 64, 16), (7, 1, 96, 48), (2, 2, 8, 16), (5, 5, 40, 32), (8, 2, 256, 16),
                                           (3, 1, 16, 128)])
def test_append_rotates_and_writes(dtype, nq, nkv, d, page):
    pos = [0, 1, page - 1, page, 3 * page - 1, 17, 2 * page, 5]
    seqs = [0, 0, 0, 0, 1, 2, 2, 1]
    _append_case(dtype, nq, nkv, d, page, 3, seqs, pos)
    _append_case(dtype, nq, nkv, d, page, 3, [1], [page + 2], theta=5e5)
    _append_case(dtype, nq, nkv, d, page, 3, seqs, pos, with_q=False)
    _append_case(dtype, nq, nkv, d, page, 3, seqs, pos, fused=False)
    in_place = _append_case(dtype, nq, nkv, d, page, 3, seqs, pos, fused=False, in_place=True)
    apart = _append_case(dtype, nq, nkv, d, page, 3, seqs, pos, fused=False)
    assert torch.equal(in_place, apart)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_leaves_out_what_has_no_place(dtype):
    """Padding, sequences and positions outside the table, pages outside the pool."""
    table = np.array([[0, 3, -1], [2, 12, 11], [-7, 2 ** 31 - 1, 4]], dtype=np.int32)          # 11 pages in the pool
    seqs = [0, -1, 0, 3, 1, 1, 2, 2, 2, -2 ** 31, 1, 0, 2]
    pos = [5, 9, 33, 4, 17, 40, 3, 20, 47, 0, -1, 48, 2 ** 31 - 1]
    _append_case(dtype, 4, 2, 64, 16, 3, seqs, pos, table=table, n_seqs=3)


def test_append_at_far_positions():
    """Angles of a position of a million turn as often as those of float64 do."""
    _append_case("f32", 4, 2, 128, 1024, 1024, [0, 0, 0, 0], [1024 * 1024 - 1, 999999, 524288, 65537], n_seqs=1)


def test_append_many_tokens():
    rng = np.random.default_rng(0)
    pos = rng.permutation(1024)[:700]
    _append_case("bf16", 6, 3, 64, 32, 32, [0] * 700, pos.tolist(), n_seqs=1)


# ---- attention --------------------------------------------------------------------------------------

class Attend:
    def __init__(self, dtype, nq, nkv, d, page, lens, seed=0, max_len=None, spare=2, stale=float("nan")):
        rng = np.random.default_rng(seed + 1)
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.nq, self.d, self.page = np.asarray(lens), nq, d, page
        self.max_len = int(self.lens.max()) if max_len is None else max_len
        need = -(-self.lens // page)
        self.n_pages = int(need.sum()) + spare
        self.max_pages = max(1, -(-self.max_len // page))
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), self.max_pages), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        k, v = (torch.randn(self.n_pages, nkv, page, d, generator=gen).to(DT[dtype]) for _ in range(2))
        for b, n in enumerate(self.lens):                # rows that were never written
            if n % page:
                k[self.table[b, n // page], :, n % page:] = stale
                v[self.table[b, n // page], :, n % page:] = stale
        for g in order[at:]:
            k[g], v[g] = stale, stale
        self.k, self.v = f64(k), f64(v)
        self.cache = sv.PagedCache(k.cuda(), v.cuda(), torch.from_numpy(self.table).cuda())
        self.q_host = 2.0 * torch.randn(len(lens), nq, d, generator=gen)
        self.q = self.q_host.cuda()
        self.seq_len = torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.out = torch.full_like(self.q, 9.0)
        self.lse = torch.full((len(lens), nq), 9.0, device="cuda")
        self.status = torch.full((len(lens),), 9, dtype=torch.int32, device="cuda")
        self.ws = torch.full((sv.sv_paged_workspace_bytes(self.cache, nq, self.max_len),), 255, dtype=torch.uint8, device="cuda")
        self.scale = 1.0 / d ** 0.5

    def call(self, window=0, sink=0, out=None):
        sv.sv_paged_attention(self.cache, self.seq_len, self.max_len, self.q, self.scale, window, sink, self.out if out is None else out,
                              self.lse, self.status, self.ws)

    def check(self, window=0, sink=0, lens=None, status=None):
        got, lse = f64(self.out.cpu()), f64(self.lse.cpu())
        q, scale, worst = f64(self.q_host), float(np.float32(self.scale)), 0.0
        for b, n in enumerate(self.lens if lens is None else lens):
            want, want_lse, reach = pc.attend(q[b], self.k, self.v, self.table[b], n, scale, window, sink)
            seen = len(pc.visible(n, window, sink))
            score = (self.d + 8) * U * reach
            weight = 2 * score + 8 * U
            rows = np.unique(self.table[b][pc.visible(n, window, sink) // self.page]) if seen else []
            rows = [g for g in rows if 0 <= g < self.n_pages]
            top = max([np.nanmax(np.abs(self.v[g])) for g in rows], default=0.0)
            tol = (weight + (seen / 4 + 64) * U) * top
            err = np.abs(got[b] - want)
            assert np.isfinite(got[b]).all() and (err <= tol).all(), (b, n, err.max(), tol)
            none = np.isneginf(want_lse)
            assert np.isneginf(lse[b][none]).all()
            lse_b, want_lse = lse[b][~none], want_lse[~none]
            assert (np.abs(lse_b - want_lse) <= score + (seen / 4 + 64) * U + 2 * U * np.abs(want_lse)).all(), (b, n)
            worst = max(worst, float((err / max(np.abs(want).max(), 1e-9)).max()))
        assert self.status.cpu().tolist() == (status or [0] * len(self.lens))
        return worst


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 281]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nkv,d,page", [(4, 4, 128, 16), (32, 8, 128, 64), (7, 1, 128, 32), (16, 1, 64, 16), (17, 1, 64, 48), (40, 2, 96, 128),
                                           (3, 3, 40, 16), (8, 2, 256, 16), (5, 5, 8, 16), (6, 2, 72, 64), (6, 3, 192, 32), (33, 1, 136, 16)])
def test_attention_of_every_small_length(dtype, nq, nkv, d, page):
    a = Attend(dtype, nq, nkv, d, page, LENS)
    a.call()
    worst = a.check()
    say(f"[paged attention {dtype} {nq}/{nkv} heads of {d}, page {page}] largest error {worst:.1e} of the row's largest value")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (16, 0), (16, 4), (17, 16), (40, 33), (100, 1), (64, 64), (257, 3), (1000, 5), (7, 1000)])
def test_attention_with_a_window(dtype, window, sink):
    """Windows and first tokens that share units of 16 rows, overlap, or reach over everything."""
    a = Attend(dtype, 6, 2, 64, 16, LENS + [600], seed=window)
    a.call(window, sink)
    a.check(window, sink)


@pytest.mark.parametrize("dtype,nq,nkv,d,page,lens", [
    ("bf16", 32, 8, 128, 256, [9001]), ("bf16", 4, 4, 64, 16, [5000, 0, 1, 4097, 300]), ("f32", 8, 2, 128, 32, [3333, 2048]),
    ("bf16", 20, 1, 256, 64, [4500, 7]), ("f32", 40, 2, 256, 16, [2500]), ("bf16", 2, 1, 96, 48, [40000])])
def test_attention_split_over_the_length(dtype, nq, nkv, d, page, lens):
    a = Attend(dtype, nq, nkv, d, page, lens)
    assert a.ws.numel() > 256                        # (that there are splits)
    for window, sink in ((0, 0), (1500, 4), (40, 3000), (2000, 0)):
        a.call(window, sink)
        worst = a.check(window, sink)
        say(f"[split {dtype} {nq}/{nkv} x {d} lengths {lens} window {window}] {worst:.1e}")


@pytest.mark.parametrize("dtype,nq,nkv,d,page,lens,window,sink", [
    ("bf16", 8, 2, 128, 16, [0, 1, 129, 191, 192, 193, 383, 384], 0, 0), ("bf16", 6, 2, 104, 32, [385, 500, 577, 600, 3], 0, 0),
    ("bf16", 4, 1, 64, 16, [0, 1, 130, 256, 257, 500, 511, 512, 513], 0, 0), ("bf16", 4, 1, 64, 64, [1100, 700, 20], 0, 0),
    ("f32", 4, 2, 48, 16, [0, 1, 65, 127, 128, 129, 250, 256, 300], 0, 0), ("f32", 16, 1, 64, 32, [900, 65, 64], 0, 0),
    ("bf16", 8, 4, 64, 16, list(range(700, 961, 4)), 0, 0), ("bf16", 16, 8, 128, 16, list(range(690, 1100, 12)), 0, 0),
    ("bf16", 16, 8, 128, 32, list(range(690, 1100, 12)), 900, 5), ("bf16", 4, 1, 64, 16, [3000, 1200, 490], 470, 20),
    ("f32", 2, 1, 64, 16, [2000, 200, 7], 230, 4), ("bf16", 32, 1, 128, 16, [380, 200, 97], 0, 0)])
def test_attention_of_workgroups_of_more_waves(dtype, nq, nkv, d, page, lens, window, sink):
    """Rows of two rounds and more, whole and in pieces, over few workgroups and over many; a page outside the pool too."""
    a = Attend(dtype, nq, nkv, d, page, lens)
    a.call(window, sink)
    a.check(window, sink)
    if window == 0:
        b = int(np.argmax(a.lens))
        a.cache.block_table[b, int(a.lens[b] - 1) // page] = a.n_pages
        a.call()
        assert a.status.cpu().tolist() == [int(i == b) for i in range(len(lens))]
        keep = a.table[b].copy()
        a.table[b, int(a.lens[b] - 1) // page:] = -1
        short = list(a.lens)
        short[b] = int(a.lens[b] - 1) // page * page
        a.check(lens=short, status=[int(i == b) for i in range(len(lens))])
        a.table[b] = keep


def test_attention_with_a_bound_above_the_lengths():
    """max_len is a bound: shorter sequences, lengths above it (clamped) and below zero."""
    a = Attend("bf16", 8, 2, 128, 16, [100, 2000, 1500, 700])
    want = a.lens.copy()
    a.seq_len[0], want[0] = -5, 0
    a.seq_len[1] = 2 ** 31 - 1
    a.call()
    a.check(lens=want)
    b = Attend("bf16", 8, 2, 128, 16, [3, 20], max_len=4000)
    b.call()
    b.check()


def test_attention_leaves_pages_outside_the_pool_out():
    for lens, max_len in (([100, 90, 300, 33], None), ([100, 90, 300, 33], 5000)):
        a = Attend("bf16", 4, 2, 64, 16, lens, max_len=max_len)
        a.table[0, 2], a.table[2, 0], a.table[2, 18], a.table[3, :3] = a.n_pages, -1, 2 ** 31 - 1, -9
        a.cache.block_table.copy_(torch.from_numpy(a.table))
        a.call()
        a.check(status=[1, 0, 1, 1])
        assert (a.out[3] == 0).all()
        a.call(window=40)                            # the bad pages of the long ones lie outside the window, one inside
        a.check(40, 0, status=[0, 0, 1, 1])


def test_attention_of_large_and_equal_scores():
    """Scores of thousands, and a maximum that comes last or first: no overflow, no lost rows."""
    for seed, size in ((0, 100.0), (1, 1e-3)):
        a = Attend("bf16", 8, 2, 128, 16, [500, 33, 1], seed=seed)
        a.q_host *= size
        a.q.copy_(a.q_host)
        a.call()
        a.check()
    a = Attend("f32", 4, 1, 64, 16, [700])
    a.cache.k.nan_to_num_(0.0)
    a.cache.k.fill_(0.5)
    a.k[:] = 0.5
    a.call()
    a.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_reaches_only_the_heads_that_read_it(dtype):
    a = Attend(dtype, 8, 4, 128, 16, [200, 90, 2000])
    clean = a.out.clone()
    a.call()
    clean.copy_(a.out)
    a.cache.v[a.table[0, 3], 1, 5, 7] = float("nan")
    a.cache.k[a.table[2, 100], 2, 0, 0] = float("inf")
    a.call()
    same = (a.out == clean).all(-1).cpu().numpy()
    for s, hs in ((0, (2, 3)), (2, (4, 5))):
        for h in range(8):
            assert same[s, h] or h in hs
    assert same[1].all() and torch.isnan(a.out[0, 2:4, 7]).all()


def test_attention_output_over_its_queries_and_reproducible():
    for lens in ([300, 20], [6000, 50]):
        a = Attend("bf16", 12, 4, 128, 32, lens)
        a.call()
        want = a.out.clone()
        for _ in range(3):
            a.ws.fill_(173)
            a.call()
            assert torch.equal(a.out, want)
        a.call(out=a.q)
        assert torch.equal(a.q, want)


def test_lse_joins_parts_of_a_cache():
    """Attention over two halves, joined by their lse, is attention over the whole."""
    a = Attend("f32", 8, 2, 64, 16, [320, 160])
    a.call()
    whole, parts = a.out.clone(), []
    table = a.cache.block_table.clone()
    for cols, lens in ((slice(0, 10), [160, 80]), (slice(10, 20), [160, 80])):
        t = table.clone()
        t[0, :10] = table[0, cols]
        t[1, :5] = table[1, 0:5] if cols.start == 0 else table[1, 5:10]
        a.cache.block_table.copy_(t)
        a.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        a.call()
        parts.append((a.out.double(), a.lse.double()))
    lse = torch.logaddexp(parts[0][1], parts[1][1])
    both = sum(o * torch.exp(l - lse)[..., None] for o, l in parts)
    assert float((both - whole).abs().max()) < 1e-5 * float(whole.abs().max())


def test_paged_calls_in_a_graph_follow_their_inputs():
    """Append and split attention recorded once, replayed with new tokens, positions and lengths."""
    a = Attend("bf16", 8, 2, 128, 16, [3000, 1200, 40], stale=0.25, max_len=3200)
    n_kv, d = 2, 128
    qkv = torch.zeros(3, 12 * d, device="cuda")
    q, k, v = (qkv[:, i * d:j * d].unflatten(1, (j - i, d)) for i, j in ((0, 8), (8, 10), (10, 12)))
    seq = torch.arange(3, dtype=torch.int32, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")

    def step():
        sv.sv_paged_append(a.cache, seq, pos, q, k, v, a.q, 1e4)
        a.call(800, 4)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    gen = torch.Generator().manual_seed(1)
    for rep in range(4):
        lens = torch.tensor([3000 - 700 * rep, 1200 - rep, 40 - rep], dtype=torch.int32)
        qkv.copy_(torch.randn(3, 12 * d, generator=gen))
        pos.copy_(lens - 1)
        a.seq_len.copy_(lens)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (a.out, a.lse, a.q, a.cache.k, a.cache.v)]
        a.out.fill_(7.0)
        a.q.fill_(7.0)
        a.ws.fill_(31)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (a.out, a.lse, a.q, a.cache.k, a.cache.v)))


def test_attention_on_another_stream_than_the_current_one():
    a = Attend("bf16", 8, 2, 64, 16, [900, 5000])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sv.sv_paged_attention(a.cache, a.seq_len, a.max_len, a.q, a.scale, 0, 0, a.out, a.lse, a.status, a.ws, stream=side)
    side.synchronize()
    a.check()


def test_offsets_beyond_32_bits():
    """A pool whose pages begin behind 2^32 bytes and 2^31 elements."""
    page, nkv, d = 1024, 8, 128
    n_pages = 2200                                   # 2.3e9 elements
    k, v = (torch.empty(n_pages, nkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.tensor([[2199, 3], [2198, 2197]], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(0)
    for g in (2199, 3, 2198, 2197):
        k[g] = torch.randn(nkv, page, d, generator=gen, device="cuda").to(torch.bfloat16)
        v[g] = torch.randn(nkv, page, d, generator=gen, device="cuda").to(torch.bfloat16)
    big = sv.PagedCache(k, v, table)
    small = sv.PagedCache(k[[2199, 3, 2198, 2197]].contiguous(), v[[2199, 3, 2198, 2197]].contiguous(),
                          torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda"))
    new = torch.randn(2, 3 * nkv, d, generator=gen, device="cuda")
    lens = torch.tensor([2000, 1025], dtype=torch.int32, device="cuda")
    seq, outs = torch.arange(2, dtype=torch.int32, device="cuda"), []
    for cache in (big, small):
        q, out = torch.empty(2, nkv, d, device="cuda"), torch.empty(2, nkv, d, device="cuda")
        ws = torch.empty(sv.sv_paged_workspace_bytes(cache, nkv, 2000), dtype=torch.uint8, device="cuda")
        sv.sv_paged_append(cache, seq, lens - 1, new[:, :nkv], new[:, nkv:2 * nkv], new[:, 2 * nkv:], q, 1e4)
        sv.sv_paged_attention(cache, lens, 2000, q, 0.1, 0, 0, out, None, None, ws)
        outs.append(out)
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0]).all())
    for g, (cg, r) in ((3, (1, 975)), (2197, (3, 0))):
        assert torch.equal(k[g, :, r], small.k[cg, :, r])


def test_arguments_that_the_binding_refuses():
    a = Attend("bf16", 4, 2, 64, 16, [40, 50])
    good = dict(seq_len=a.seq_len, max_len=50, q=a.q, scale=0.1, window=0, n_sink=0, out=a.out, lse=a.lse, status=a.status, workspace=a.ws)
    for bad in (dict(seq_len=a.seq_len[:1]), dict(seq_len=a.seq_len.long()), dict(q=a.q.bfloat16()), dict(q=a.q[:, :, :32]),
                dict(out=a.out[:1]), dict(lse=a.lse[:1]), dict(status=a.status[:1]), dict(q=a.q.cpu()), dict(workspace=a.ws.float()),
                dict(q=a.q.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            sv.sv_paged_attention(a.cache, **{**good, **bad})
    for bad, status in ((dict(max_len=65), -2), (dict(window=-1), -2), (dict(workspace=a.ws[:128]), -5), (dict(workspace=a.ws[4:]), -5)):
        with pytest.raises(sv.SvError) as e:
            sv.sv_paged_attention(a.cache, **{**good, **bad})
        assert e.value.status == status
    k = torch.zeros(2, 2, 64, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    for args in ((pos, pos[:1], None, k, k, None), (pos, pos, k, k, k, None), (pos, pos, None, k[:1], k, None), (pos, pos, None, k, k.half(), None),
                 (pos, pos, None, k, k[:, :, :32], None), (pos.long(), pos, None, k, k, None), (pos, pos, k, k, k, k[:1])):
        with pytest.raises(ValueError):
            sv.sv_paged_append(a.cache, *args, 1e4)
    z = torch.zeros(4, 8, device="cuda")
    for p, q in ((z, z[:2]), (z, z.double()), (z[0], z[0]), (z, z.t().contiguous().t()), (z.cpu(), z)):
        with pytest.raises(ValueError):
            sv.sv_token_probs(p, 1.0, q)
    with pytest.raises(sv.SvError) as e:
        sv.sv_token_probs(z, 0.0, z)
    assert e.value.status == sv.SV_ERR_TOKEN


# ---- together ---------------------------------------------------------------------------------------

def test_verifiers_own_cache_read_as_pages():
    """The contiguous cache of a verification layer, as pages: attention of one query per episode."""
    cfg = sv.model_cfg("bf16", 512, 4, 128, 1536, 1024)
    lens = [70, 33]
    kv = sv.KvCache(cfg, 2, 96, lens)
    gen = torch.Generator().manual_seed(2)
    kv.k.copy_(torch.randn(2, 4, 96, 128, generator=gen))
    kv.v.copy_(torch.randn(2, 4, 96, 128, generator=gen))
    cache = sv.PagedCache.of_kv_cache(kv)
    q = torch.randn(2, 4, 128, generator=gen)
    out, lse = torch.empty(2, 4, 128, device="cuda"), torch.empty(2, 4, device="cuda")
    ws = torch.empty(sv.sv_paged_workspace_bytes(cache, 4, 96), dtype=torch.uint8, device="cuda")
    sv.sv_paged_attention(cache, kv.prefix_len, 70, q.cuda(), 128 ** -0.5, 0, 0, out, lse, None, ws)
    for b in range(2):
        want, _, reach = pc.attend(f64(q[b]), f64(kv.k.cpu()), f64(kv.v.cpu()), [b], lens[b], 128 ** -0.5)
        assert np.abs(f64(out[b].cpu()) - want).max() <= (2 * 136 * U * reach + 100 * U) * float(kv.v.abs().max())


def test_speculative_decoding_by_sampling():
    """The operators as they are used: a small drafter decodes a chain over its paged cache, the tree pass scores it,
    sampled acceptance decides, the verifier's cache is committed and the drafter's cut back.  Every stage against
    the oracles, on the inputs that the stage before left."""
    B, T, V, d, nq, nkv, steps = 2, 4, 256, 64, 4, 2, 4
    cfg = wl.C2.scaled(name="bf16-sampled", index=61, n_layers=2, hidden=512, n_heads=4, head_dim=128, mlp_dim=1536, vocab=1024,
                       n_bins=V, n_episodes=B, tree_nodes=T, prefix_lo=30, prefix_hi=40, max_depth=T - 1, max_children=1, spine_lo=T - 1)
    pl = wl.prefix_lengths(cfg)
    chain = np.arange(-1, T - 1)
    vp = VerifyPass(cfg, pl, np.concatenate([chain] * B), extra_capacity=steps * T)
    for l in range(cfg.n_layers):
        vp.load_layer(l, wl.layer_weights(cfg, l))
        for b in range(B):
            vp.load_prefix(l, b, *wl.prefix_kv(cfg, b, l, int(pl[b])))
    head = wl.head_weights(cfg)
    vp.load_head(head["g_final"], head["w_lm"])
    gen = torch.Generator().manual_seed(4)
    embed = torch.randn(V, cfg.hidden, generator=gen).cuda()
    w_qkv = (torch.randn(cfg.hidden, (nq + 2 * nkv) * d, generator=gen) / cfg.hidden ** 0.5).cuda()
    w_out = (torch.randn(nq * d, V, generator=gen) * 0.1).cuda()

    page, max_pages = 16, 4
    pool = [torch.zeros(B * max_pages, nkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = np.random.default_rng(0).permutation(B * max_pages).reshape(B, max_pages).astype(np.int32)
    cache = sv.PagedCache(*pool, torch.from_numpy(table).cuda())
    seq = torch.arange(B, dtype=torch.int32, device="cuda")
    length = torch.zeros(B, dtype=torch.int32, device="cuda")            # committed tokens in the drafter's cache
    ws = torch.empty(sv.sv_paged_workspace_bytes(cache, nq, page * max_pages), dtype=torch.uint8, device="cuda")
    q, out = torch.empty(B, nq, d, device="cuda"), torch.empty(B, nq, d, device="cuda")
    root = torch.randint(0, V, (B,), generator=gen).cuda()
    lo, emitted = cfg.vocab - V, [[] for _ in range(B)]
    for step in range(steps):
        say(f"[sampled decoding] step {step}")
        tok = torch.zeros(B, T, dtype=torch.int64, device="cuda")
        tok[:, 0] = root
        q_prob = torch.zeros(B, T, V, device="cuda")
        for n in range(T):                           # (the last one only leaves its keys and values)
            qkv = embed[tok[:, n]] @ w_qkv
            part = [qkv[:, i * d:j * d].unflatten(1, (j - i, d)) for i, j in ((0, nq), (nq, nq + nkv), (nq + nkv, nq + 2 * nkv))]
            sv.sv_paged_append(cache, seq, length + n, *part, q, cfg.rope_theta)
            sv.sv_paged_attention(cache, length + n + 1, page * max_pages, q, d ** -0.5, 24, 4, out, None, None, ws)
            want = [pc.attend(f64(q[b].cpu()), f64(pool[0].cpu()), f64(pool[1].cpu()), table[b], int(length[b]) + n + 1, d ** -0.5, 24, 4)
                    for b in range(B)]
            for b in range(B):
                assert np.abs(f64(out[b].cpu()) - want[b][0]).max() <= (2 * (d + 8) * U * want[b][2] + 90 * U) * float(pool[1].abs().max())
            logits = out.flatten(1) @ w_out
            row = torch.empty_like(logits)
            sv.sv_token_probs(logits, 0.8, row)
            q_prob[:, n] = row
            if n + 1 < T:
                u = torch.rand(B, generator=gen).cuda()
                tok[:, n + 1] = (row.double().cumsum(1) <= (u.double() * row.double().sum(1))[:, None]).sum(1).clamp(max=V - 1)
        vp.set_hidden(embed[tok.reshape(-1)] * 0.2)
        vp.set_draft((tok + lo).cpu().numpy())
        vp.forward(want_logits=True)
        u_accept, u_draw = torch.rand(B * T, generator=gen), torch.rand(B, generator=gen)
        vp.accept_sampled(u_accept.cuda(), u_draw.cuda(), 0.8, q_prob.view(B * T, V))
        _check_probs(f64(vp.probs.cpu()), f64(vp.logits.cpu()), float(np.float32(0.8)))
        for b in range(B):
            rows = slice(b * T, (b + 1) * T)
            ref = sa.sampled_accept(chain, (tok[b] + lo).tolist(), f64(vp.probs[rows].cpu()), f64(q_prob[b].cpu()), lo,
                                    f64(u_accept[rows]), float(u_draw[b]), T - 1)
            n = ref["length"]
            assert int(vp.accepted_len[b]) == n and vp.out_tokens[b, :n + 1].tolist() == ref["tokens"] and int(vp.accept_status[b]) == 0
            emitted[b] += ref["tokens"]
        prefix = vp.kv[0].prefix_len.clone()
        vp.commit()
        assert torch.equal(vp.kv[0].prefix_len, prefix + vp.accepted_len + 1)
        length += vp.accepted_len + 1                # the rejected rows are overwritten by what follows
        root = vp.out_tokens.gather(1, vp.accepted_len.long()[:, None])[:, 0].long() - lo
    say(f"[sampled decoding] {steps} steps emitted {[len(e) for e in emitted]} tokens")
    assert all(len(e) >= steps for e in emitted)


@pytest.mark.parametrize("rows", [1, 5, 33, 100, 130])
def test_token_probs_of_long_rows_in_shares(rows):
    """Rows too long for the registers, few enough that several workgroups write one; the same in place."""
    gen = torch.Generator().manual_seed(rows)
    z = 5 * torch.randn(rows, 40961, generator=gen)
    z[rows // 2, 40000:] = -float("inf")
    d = z.cuda()
    p = torch.full((rows, 40961), -1.0, device="cuda")
    sv.sv_token_probs(d, 0.9, p)
    _check_probs(f64(p.cpu()), f64(z), float(np.float32(0.9)))
    sv.sv_token_probs(d, 0.9, d)
    assert torch.equal(d, p)


# ---- forms and borders that the sizes above do not reach -------------------------------------------

@pytest.mark.parametrize("rows", [1, 5])
@pytest.mark.parametrize("n", [8192, 8193, 32768, 32769])
def test_token_probs_where_the_kernel_changes(rows, n):
    """The last column of a thread's registers, and the first that they do not hold."""
    test_token_probs(rows, n)


@pytest.mark.parametrize("n", [5, 300, 3000, 20000, 40000])
def test_token_probs_at_the_ends_of_the_range(n):
    """Temperatures from the smallest to the largest, logits whose differences float32 does not hold."""
    gen = torch.Generator().manual_seed(n)
    for t in (5e-39, 2e-38, 1e-30, 0.999, 1.0, 1.001, 1e30, 1e37, 1e38, 3e38):
        z = (torch.randn(6, n, generator=gen) * max(t, 1.0)).clamp(-3.4e38, 3.4e38)
        z[0] = -float("inf")
        z[1, 1:] = -float("inf")
        z[2, ::2] = torch.finfo(torch.float32).min
        z[3], z[3, ::3] = 3.4e38, -3.4e38
        z[4] *= 1e-30
        d = z.cuda()
        p = torch.empty_like(d)
        sv.sv_token_probs(d, t, p)
        _check_probs(f64(p.cpu()), f64(z), float(np.float32(t)))
        sv.sv_token_probs(d, t, d)
        assert torch.equal(d, p)


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [40, 300, 5000, 20000, 40000])
def test_rows_off_the_walk_have_no_effect(V, drawn):
    """Rows of nodes that the walk did not come to hold NaN, infinity or mass everywhere: the same outputs."""
    rng = np.random.default_rng(V)
    B, T = 4, 20
    a = Accept(_trees(B, T, 5, 3, rng), 5)
    p, q = _probs(rng, (B, T, V), 1.0), _probs(rng, (B, T, V), 1.0) * 0.3 + _probs(rng, (B, T, V), 1.0) * np.float32(0.7)
    tok = _draft_tokens(a.parents, p.astype(float), rng, drawn)
    p, q = (torch.from_numpy(x.astype(np.float32)).cuda() for x in (p, q))
    tok = torch.from_numpy(tok.reshape(-1)).int().cuda()
    u, ud = torch.from_numpy(0.2 * rng.random(B * T)).float().cuda(), torch.from_numpy(rng.random(B)).float().cuda()
    call = lambda: a.call(tok, p.view(B * T, V), q.view(B * T, V) if drawn else None, 0, u, ud)
    keep = p.clone(), q.clone()
    for first in (False, True):                      # by these numbers, and down to a leaf by each node's first child
        if first:
            u.zero_()
        p.copy_(keep[0])
        q.copy_(keep[1])
        call()
        want = [t.clone() for t in a.outputs()]
        on = a.mask.view(B, T).bool()
        assert bool((on.sum(1) < T).all()) and (not first or int(a.length.min()) > 0)
        for junk in (float("nan"), float("inf"), 1e30, -1.0):
            p[~on] = junk
            q[~on] = junk
            call()
            assert all(torch.equal(x, y) for x, y in zip(want, a.outputs()))


MANY = [i * 7 % 40 for i in range(60)] + [1290, 800, 500, 1000, 64]


# more rows planned (sequences x units that max_len and the window allow) than the Infinity Cache holds: loads past the caches
@pytest.mark.parametrize("dtype,nq,nkv,d,page,lens,max_len,window,sink", [
    ("bf16", 8, 4, 64, 16, [0, 1, 17, 300, 1700, 2500], 90000, 0, 0), ("f32", 4, 4, 48, 32, [2500, 0, 129, 600], 90000, 0, 0),
    ("bf16", 32, 8, 128, 64, [1, 700, 0, 3000], 60000, 0, 0), ("f32", 6, 2, 96, 16, [33, 1900, 5], 120000, 0, 0),
    ("bf16", 16, 1, 256, 16, [2100, 40], 140000, 0, 0), ("f32", 3, 3, 192, 48, [15, 1000, 2000], 60000, 0, 0),
    # whole rows, of which a workgroup has more rounds than it would take more waves for
    ("bf16", 16, 16, 64, 16, MANY, 1290, 0, 0), ("bf16", 16, 16, 128, 32, MANY, 1290, 0, 0),
    ("f32", 16, 16, 64, 16, MANY, 1290, 0, 0),
    # a window, of rows in pieces and whole
    ("bf16", 6, 2, 128, 16, [0, 3000, 900, 2000, 1], 100000, 99000, 5), ("bf16", 16, 16, 128, 16, MANY, 2000, 650, 20),
    ("f32", 32, 16, 64, 16, MANY, 2000, 600, 33), ("f32", 16, 16, 256, 16, [n % 700 for n in MANY], 900, 530, 4)])
def test_attention_past_the_caches(dtype, nq, nkv, d, page, lens, max_len, window, sink):
    """Every type and size of head; with a page outside the pool too."""
    units = -(-max_len // 16)
    if window:
        units = min(units, -(-sink // 16) + -(-window // 16) + 1)
    assert len(lens) * units * 16 * 2 * nkv * d * (4 if dtype == "f32" else 2) > 256 << 20 and nq // nkv <= 16
    a = Attend(dtype, nq, nkv, d, page, lens, max_len=max_len)
    a.call(window, sink)
    worst = a.check(window, sink)
    say(f"[past the caches {dtype} {nq}/{nkv} x {d} max_len {max_len} window {window}] {worst:.1e}")
    b = int(np.argmax(a.lens))
    a.table[b, int(a.lens[b] - 1) // page] = a.n_pages
    a.cache.block_table.copy_(torch.from_numpy(a.table))
    a.call(window, sink)
    a.check(window, sink, status=[int(i == b) for i in range(len(lens))])
