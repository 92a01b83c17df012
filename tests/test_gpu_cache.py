"""The growing cache on the GPU against the float64 oracle: writes, reads, pool writes and
the attention of chunks, at the sizes, layouts and lengths where they can go wrong.

Tolerances.  A value rounded once to bf16 is off by at most 2^-8 of itself; a turned key is
x c - y s of fp32 cos and sin (each within 2^-22) and fp32 products, off by at most
2^-21 (|x| + |y|) before that rounding.  An int8 code is off by half a scale, the scale by
2^-22 of itself (a maximum of such keys, one division); its decoded value is rounded to
bf16.  Attention: the bar of the other parity tests (fp32 1e-5; bf16 and int8 2e-2 with a
mean of 1e-2, lse 5e-2), and for bf16 a 2-norm of the error of 1e-2 of the output's: query
and probability rounding are each at most 2^-8 relative a term, and their errors are
independent over terms."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_17715_amd as c2kv
import synth
from cache_common import ACT, Scene, f64
from gpu_common import Dev, say
from oracle import cache_oracle

pytestmark = pytest.mark.gpu

STORES = ["f32", "bf16", "i8"]


def near_rounded(got, ref, amp, act, extra=0.0):
    """got: the act type's rounding of fp32 values within 2^-21 amp of ref."""
    half = 2.0 ** -24 if act == torch.float32 else 2.0 ** -8
    err = np.abs(got - ref)
    bound = half * np.abs(ref) + 2.0 ** -21 * amp + extra
    assert (err <= bound * (1 + 1e-6) + 1e-30).all(), float((err - bound).max())


def amplitude(x):
    h = x.shape[-1] // 2
    a = np.abs(x[..., :h]) + np.abs(x[..., h:])
    return np.concatenate([a, a], -1)


SHAPES = [
    # one token a request, odd heads
    dict(n=[1, 1, 1], ctx=[0, 63, 200], hq=6, hkv=3),
    # a few tokens a request, some without any, chunks over a tile and a page edge
    dict(n=[3, 0, 8, 1], ctx=[62, 5, 124, 0], page=128, fused=True),
    # longer chunks than the row kernel takes: tiles that begin and end inside
    dict(n=[70, 1, 0, 130], ctx=[10, 64, 3, 127], fused=True, pad_rows=3),
    dict(n=[64, 64], ctx=[0, 64], d=64, hq=4, hkv=4, page=128),
    dict(n=[257], ctx=[61], hq=2, hkv=1, page=192, d=64, far=1_000_000),
    dict(n=[2] * 70 + [9], ctx=list(range(71)), hq=2, hkv=1, d=64),
    # more (token, head) pairs than run at once: tiles for longer chunks, rows for hinted ones
    dict(n=[300, 1, 0, 77, 64, 129], ctx=[10, 64, 3, 127, 5, 62], hkv=8, fused=True, pad_rows=3),
    dict(n=[700, 33], ctx=[61, 100], hkv=4, d=64, page=192, far=1_000_000),
    dict(n=[64] * 33 + [5], ctx=list(range(34)), hq=3, hkv=1),
]


@pytest.mark.parametrize("hint", [0, 1, 1000])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_write(i, store, hint):
    s = Scene(store, seed=i, **SHAPES[i])
    say(f"write {store} {SHAPES[i]} hint {hint}")
    before = s.copies()
    rope = i % 2 == 0 or store == "i8"
    pos = s.pos if rope else None
    # hints choose the kernel: each must give the same
    c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(max_chunk=hint), s.k, s.v, pos)
    torch.cuda.synchronize()
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    assert len(where) == s.tok_off[-1] > 0
    k64 = cache_oracle.turned(f64(s.k), s.pos.cpu().numpy() if rope else None, s.base)
    v64 = f64(s.v)
    rows = np.array(sorted(where))
    page = np.array([where[r][2] for r in rows])
    at = np.array([where[r][3] for r in rows])
    kp, vp = f64(s.kp), f64(s.vp)
    gk, gv = kp[page, :, at], vp[page, :, :, at]
    if store == "i8":
        for got, scale, x, amp in ((gk, f64(s.ks), k64[rows], amplitude(f64(s.k))[rows]),
                                   (gv, f64(s.vs), v64[rows], 0 * v64[rows])):
            sc = scale[page, :, at]
            ref = cache_oracle.int8_scale(x)
            slack = 2.0 ** -21 * amp.max(-1) / 127
            assert (np.abs(sc - ref) <= 2.0 ** -22 * ref + slack).all()
            err = np.abs(got * sc[..., None] - x)
            bound = 0.5 * sc[..., None] * (1 + 2.0 ** -14) + 2.0 ** -21 * amp
            assert (err <= bound).all(), float((err - bound).max())
            assert np.abs(got).max() <= 127 and (np.abs(got).max(-1) == 127).all()
    else:
        if rope:
            near_rounded(gk, k64[rows], amplitude(f64(s.k))[rows], s.act)
        else:
            np.testing.assert_array_equal(gk, k64[rows])
        np.testing.assert_array_equal(gv, v64[rows])
    # everything else in the cache is as it was
    for now, was, value in ((s.kp, before[0], False), (s.vp, before[1], True),
                            (s.ks, before[2], None), (s.vs, before[3], None)):
        if now is None:
            continue
        now, was = now.clone(), was.clone()
        pt, at_t = torch.from_numpy(page).cuda(), torch.from_numpy(at).cuda()
        for t in (now, was):
            if value:
                t[pt, :, :, at_t] = 0
            else:
                t[pt, :, at_t] = 0
        assert torch.equal(now, was)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("n", [[1] * 300, [0] * 50 + [200] + [0] * 249])
def test_write_of_a_step_without_a_bound(n, store):
    """No more tokens than requests go by rows, a long chunk among them as well: the same as under
    every bound."""
    s = Scene(store, n, [(7 * i) % 150 for i in range(300)], hq=8, hkv=8, d=64, seed=36)
    before, after = s.copies(), []
    for hint in (0, 1, 300):
        for t, was in zip((s.kp, s.vp, s.ks, s.vs), before):
            if t is not None:
                t.copy_(was)
        c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(max_chunk=hint), s.k, s.v, s.pos)
        after.append(s.copies())
    torch.cuda.synchronize()
    assert not torch.equal(before[0], after[0][0])
    for other in after[1:]:
        assert all(a is None or torch.equal(a, b) for a, b in zip(after[0], other))


@pytest.mark.parametrize("turn", [False, True])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_read(i, store, turn):
    s = Scene(store, seed=20 + i, **SHAPES[i])
    say(f"read {store} {SHAPES[i]} turn {turn}")
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    k = torch.full((s.n_tokens, s.hkv, s.d), 7.0, dtype=s.act, device="cuda")
    v = torch.full_like(k, 7.0)
    t = (5 - s.pos) if turn else None
    c2kv.c2kv_cache_read(s.cfg, s.cache, s.chunks(), k, v, t)
    torch.cuda.synchronize()
    kp, vp = s.pages64()
    rows = np.array(sorted(where))
    page = np.array([where[r][2] for r in rows])
    at = np.array([where[r][3] for r in rows])
    k0, v0 = kp[page, :, at], vp[page, :, :, at]
    ref = cache_oracle.turned(k0, t.cpu().numpy()[rows] if turn else None, s.base)
    near_rounded(f64(k)[rows], ref, amplitude(k0), s.act)
    near_rounded(f64(v)[rows], v0, np.abs(v0) * (store == "i8"), s.act)
    rest = np.setdiff1d(np.arange(s.n_tokens), rows)
    assert (k[rest] == 7.0).all() and (v[rest] == 7.0).all()


def test_int8_rows_of_zeros_infinities_and_nans():
    """A row of zeros comes back as zeros, one with an infinity or a NaN as NaN; the rows
    beside it are not touched by it."""
    s = Scene("i8", [70], [10], hq=2, hkv=2)
    k, v = s.k.clone(), s.v.clone()
    k[0], v[1] = 0, 0
    k[2, 0, 5], v[3, 1, 77], k[4, 1, 100] = float("inf"), float("nan"), float("-inf")
    for hint in (1, 100):
        c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(max_chunk=hint), k, v)
        rk, rv = torch.empty_like(k), torch.empty_like(v)
        c2kv.c2kv_cache_read(s.cfg, s.cache, s.chunks(), rk, rv)
        torch.cuda.synchronize()
        assert (rk[0] == 0).all() and (rv[1] == 0).all()
        for t, i, h in ((rk, 2, 0), (rv, 3, 1), (rk, 4, 1)):
            assert not torch.isfinite(t[i, h]).any()
            assert torch.isfinite(t[i, 1 - h]).all()
        assert torch.isfinite(rk[5:]).all() and torch.isfinite(rv[4:]).all()


def test_int8_tiles_of_zeros_infinities_and_nans():
    s = Scene("i8", [1200], [7], seed=4)
    s.k[3] = 0
    s.k[500, 1, 5] = float("inf")
    s.v[501, 0, 9] = float("nan")
    s.v[502, 0] = 2.0 ** -110
    c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(), s.k, s.v)
    torch.cuda.synchronize()
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    kp, vp = s.pages64()
    key = lambda i, h: kp[where[i][2], h, where[i][3]]
    value = lambda i, h: vp[where[i][2], h, :, where[i][3]]
    assert (key(3, 0) == 0).all() and (key(3, 1) == 0).all()
    assert np.isnan(key(500, 1)).all() and np.isfinite(key(500, 0)).all()
    assert np.isnan(value(501, 0)).all() and np.isfinite(value(501, 1)).all()
    assert (value(502, 0) == 0).all() and (value(502, 1) != 0).any()


@pytest.mark.parametrize("how", ["rows", "tiles", "pool"])
def test_int8_codes_are_the_rounded_quotients(how):
    """scale = max / 127 and code = x / scale, each one fp32 division rounded once, the code then
    to the nearest whole number (halves to even): bit for bit, for every pair of bf16 mantissas
    over ten powers of two.  (Half of a row's maximum is such a half, 63.5, but for the
    scale's own rounding.)"""
    m = np.arange(128, 256, dtype=np.float32) / 128
    top = np.repeat(m, 10)                       # a row for each maximum and power of two
    x = np.tile(np.exp2(-np.arange(10, dtype=np.float32)), 128)[:, None] * m[None]
    x[:, 1::2] *= -1
    x = np.where(np.abs(x) > top[:, None], 0, x).astype(np.float32)
    x[np.arange(len(x)), np.arange(len(x)) % 128] = top
    scale = top / np.float32(127)
    code = np.rint(x / scale[:, None])
    assert scale.dtype == code.dtype == np.float32
    n = len(x)
    cfg = c2kv.attn_cfg(1, 1, 128, "bf16", 1e4)
    rows = torch.from_numpy(x).cuda().bfloat16()[:, None]
    assert (rows[:, 0].float().cpu().numpy() == x).all()
    if how == "pool":
        pk, pv = (torch.zeros((n, 1, 128), dtype=torch.int8, device="cuda") for _ in range(2))
        ks, vs = (torch.zeros((n, 1), device="cuda") for _ in range(2))
        c2kv.c2kv_pool_write(cfg, c2kv.pool_desc(pk, pv, ks, vs),
                             torch.arange(n, device="cuda"), rows, rows.flip(0))
        got = [t[:, 0].cpu().numpy() for t in (pk, ks, pv.flip(0), vs.flip(0))]
    else:
        # 1280 units go by rows, those of two heads by tiles
        heads = 1 if how == "rows" else 2
        s = Scene("i8", [n], [5], hq=heads, hkv=heads)
        rows = rows.expand(n, heads, 128).contiguous()
        c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(), rows, rows.flip(0))
        where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, n)
        page, at = (np.array([where[r][i] for r in range(n)]) for i in (2, 3))
        got = [s.kp.cpu().numpy()[page, -1, at], s.ks.cpu().numpy()[page, -1, at],
               s.vp.cpu().numpy()[page, -1, :, at][::-1], s.vs.cpu().numpy()[page, -1, at][::-1]]
    for c, sc in (got[:2], got[2:]):
        np.testing.assert_array_equal(sc, scale)
        np.testing.assert_array_equal(c, code)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("n,d,hkv", [(1, 128, 8), (33, 64, 3), (1000, 128, 2), (257, 64, 1)])
def test_pool_write(n, d, hkv, store):
    say(f"pool write {store} n={n} d={d} hkv={hkv}")
    s = Scene(store, [n], [0], hq=2 * hkv, hkv=hkv, d=d, seed=n, fused=True)
    rows = n + 5
    g = torch.Generator().manual_seed(n)
    row = torch.randperm(rows, generator=g)[:n]
    if n > 30:                                   # rows outside the pool are skipped
        row[3], row[9], row[30] = -1, rows, 1 << 40
    kept = [i for i in range(n) if 0 <= row[i] < rows]
    pk = torch.full((rows, hkv, d), 3, dtype=s.kp.dtype, device="cuda")
    pv = torch.full_like(pk, 3)
    ks = vs = None
    if store == "i8":
        ks = torch.full((rows, hkv), 3.0, device="cuda")
        vs = ks.clone()
    pool = c2kv.pool_desc(pk, pv, ks, vs)
    c2kv.c2kv_pool_write(s.cfg, pool, row.cuda(), s.k, s.v, s.pos)
    torch.cuda.synchronize()
    r = row[kept].numpy()
    x = f64(s.k)[kept]
    k64 = cache_oracle.turned(x, s.pos.cpu().numpy()[kept], s.base)
    v64 = f64(s.v)[kept]
    if store == "i8":
        for codes, sc, ref, amp in ((f64(pk)[r], f64(ks)[r], k64, amplitude(x)),
                                    (f64(pv)[r], f64(vs)[r], v64, 0 * v64)):
            assert (np.abs(sc - cache_oracle.int8_scale(ref)) <=
                    2.0 ** -22 * sc + 2.0 ** -21 * amp.max(-1) / 127).all()
            err = np.abs(codes * sc[..., None] - ref)
            assert (err <= 0.5 * sc[..., None] * (1 + 2.0 ** -14) + 2.0 ** -21 * amp).all()
    else:
        near_rounded(f64(pk)[r], k64, amplitude(x), s.act)
        np.testing.assert_array_equal(f64(pv)[r], v64)
    rest = np.setdiff1d(np.arange(rows), r)
    assert (pk[rest] == 3).all() and (pv[rest] == 3).all()
    if store == "i8":
        assert (ks[rest] == 3).all() and (vs[rest] == 3).all()


# ---- attention ------------------------------------------------------------------

def check_attend(s, out, lse, ref, ref_lse, has):
    o, l = f64(out), f64(lse)
    assert (o[~has] == 7.0).all() and (l[~has] == 7.0).all()
    o, l, ref, ref_lse = o[has], l[has], ref[has], ref_lse[has]
    empty = np.isneginf(ref_lse)
    assert (np.isneginf(l) == empty).all()
    assert (o[empty] == 0).all()
    assert np.isfinite(o).all() and np.isfinite(l[~empty]).all()
    err, lerr = np.abs(o - ref), np.abs(l[~empty] - ref_lse[~empty])
    say(f"max {err.max():.2e} mean {err.mean():.2e} lse {lerr.max() if lerr.size else 0:.2e}")
    if s.store == "f32":
        assert err.max() <= 1e-5 and (not lerr.size or lerr.max() <= 1e-5)
    else:
        assert err.max() <= 2e-2 and err.mean() <= 1e-2
        assert not lerr.size or (lerr.max() <= 5e-2 and lerr.mean() <= 1e-2)
        assert np.linalg.norm(o - ref) <= 1e-2 * np.linalg.norm(ref) + 1e-30


def dense64(s, q, pos, lens=None):
    """The oracle's attention by float64 matrix products on the GPU, for larger scenes
    (every page there)."""
    kp, vp = s.pages64()
    out = np.zeros((s.n_tokens, s.hq, s.d))
    lse = np.full((s.n_tokens, s.hq), -np.inf)
    has = np.zeros(s.n_tokens, bool)
    qt = cache_oracle.turned(f64(q), pos, s.base)
    G = s.hq // s.hkv
    for b in range(s.B):
        r0, r1, n = int(s.tok_off[b]), int(s.tok_off[b + 1]), int(s.kv_len[b])
        has[r0:r1] = True
        if n == 0:
            continue
        ids = s.table[b][:-(-n // s.page)]
        k = torch.from_numpy(np.concatenate([kp[i] for i in ids], 1)[:, :n]).cuda()
        v = torch.from_numpy(np.concatenate([vp[i] for i in ids], 2)[:, :, :n]).cuda()
        j = torch.arange(n, device="cuda")
        hidden = j[None] > (n - (r1 - r0) + torch.arange(r1 - r0, device="cuda"))[:, None]
        for h in range(s.hq):
            x = torch.from_numpy(qt[r0:r1, h]).cuda() @ k[h // G].T.contiguous() / s.d ** 0.5
            x = x.masked_fill(hidden, -torch.inf)
            out[r0:r1, h] = (torch.softmax(x, -1) @ v[h // G].T.contiguous()).cpu().numpy()
            lse[r0:r1, h] = torch.logsumexp(x, -1).cpu().numpy()
    return out, lse, has


ATTEND = [
    dict(n=[1], ctx=[0]),                                     # one token that sees itself
    dict(n=[1, 1, 1], ctx=[0, 63, 64], hq=4, hkv=4),          # tile edges, one head a kv-head
    dict(n=[1] * 5, ctx=[31, 500, 1, 700, 129], hq=8, hkv=1, page=128),
    dict(n=[1, 1], ctx=[1000, 3], hq=21, hkv=3, d=64, page=192),      # seven heads a kv-head
    dict(n=[1], ctx=[900], hq=48, hkv=2),                     # 24 heads: more than 16 rows
    dict(n=[3, 5, 1, 7], ctx=[700, 61, 0, 130], hq=8, hkv=2, fused=True),
    dict(n=[2, 0, 4], ctx=[300, 40, 62], hq=16, hkv=1, d=64), # 32 to 64 rows
    dict(n=[9, 17], ctx=[100, 260], hq=12, hkv=4, d=64, pad_rows=2),
    dict(n=[33, 64, 1], ctx=[0, 77, 400], hq=4, hkv=2, page=256, fused=True),
    dict(n=[130], ctx=[0], hq=4, hkv=1),
    dict(n=[65, 3], ctx=[190, 640], hq=8, hkv=2, d=64),
    dict(n=[200], ctx=[57], hq=3, hkv=3, page=128),
    dict(n=[1] * 130, ctx=[(7 * i) % 150 for i in range(130)], hq=2, hkv=1, d=64),
]


@pytest.mark.parametrize("hint", [False, True])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("i", range(len(ATTEND)))
def test_attend(i, store, hint):
    s = Scene(store, seed=40 + i, **ATTEND[i])
    say(f"attend {store} {ATTEND[i]} hint {hint}")
    kw = dict(max_chunk=max(s.n), max_kv=int(s.kv_len.max())) if hint else {}
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(**kw), s.q, out, s.pos, lse)
    torch.cuda.synchronize()
    check_attend(s, out, lse, *dense64(s, s.q, s.pos.cpu().numpy()))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("shape", [
    dict(n=[1, 1], ctx=[7000, 129], hq=8, hkv=2),             # one long request, one short
    dict(n=[1] * 40, ctx=[300 + 13 * i for i in range(40)], hq=8, hkv=8, d=64),
    dict(n=[6, 6, 6], ctx=[3000, 10, 1500], hq=16, hkv=2),
    dict(n=[300, 1, 40], ctx=[2000, 4000, 0], hq=8, hkv=2),
    dict(n=[1100], ctx=[0], hq=4, hkv=2, d=64),
    dict(n=[700], ctx=[900], hq=8, hkv=1),
])
def test_attend_larger(shape, store):
    s = Scene(store, seed=77, **shape)
    say(f"attend {store} {shape}")
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(max_chunk=max(s.n)), s.q, out, s.pos, lse)
    torch.cuda.synchronize()
    check_attend(s, out, lse, *dense64(s, s.q, s.pos.cpu().numpy()))


@pytest.mark.parametrize("hints", [dict(max_chunk=1), dict(max_chunk=1, max_kv=1),
                                   dict(max_chunk=2), dict(max_chunk=10_000, max_kv=1 << 30)])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("i", [4, 5, 9])
def test_bounds_that_do_not_hold_change_no_result(i, store, hints):
    """max_chunk and max_kv choose launch shapes: chunks and caches beyond them are answered
    as well (24 heads a kv-head of one token; ragged drafts; 130 tokens)."""
    s = Scene(store, seed=60 + i, **ATTEND[i])
    say(f"attend {store} {ATTEND[i]} {hints}")
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(**hints), s.q, out, s.pos, lse)
    torch.cuda.synchronize()
    check_attend(s, out, lse, *dense64(s, s.q, s.pos.cpu().numpy()))


@pytest.mark.parametrize("store", ["bf16", "i8"])
@pytest.mark.parametrize("hint,half,blocks", [
    (1, 2.0 ** -16, False),                      # single tokens: two bf16 numbers a query
    (5, 2.0 ** -16, True), (32, 2.0 ** -16, True),           # blocks of 128 rows: the same
    (33, 2.0 ** -8, True), (0, 2.0 ** -8, True),             # of 256 rows: one
])
def test_bounds_choose_how_far_queries_are_rounded(hint, half, blocks, store):
    """The header's figures.  A score is off by at most `half` of the sum of its products'
    magnitudes, and by what fp32 makes of turns and sums (2^-20 of it); the log-sum-exp is off by
    no more, and in blocks, which sum the probabilities that they rounded to bf16, by 2^-8."""
    s = Scene(store, [5, 3], [700, 90], pad_rows=50, seed=35)
    out, lse = s.out(), s.lse()
    ch = s.chunks(max_chunk=hint)
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, s.q, out, s.pos, lse)
    torch.cuda.synchronize()
    ref, ref_lse, has = dense64(s, s.q, s.pos.cpu().numpy())
    check_attend(s, out, lse, ref, ref_lse, has)
    # the largest sum of magnitudes of a (token, head)'s scores, from the pairs' amplitudes
    amp, G = amplitude(f64(s.q)), s.hq // s.hkv
    kp = np.abs(s.pages64()[0])
    worst = np.zeros((s.n_tokens, s.hq))
    for b in range(s.B):
        r0, r1, n = int(s.tok_off[b]), int(s.tok_off[b + 1]), int(s.kv_len[b])
        k = np.concatenate([kp[i] for i in s.table[b][:-(-n // s.page)]], 1)[:, :n]
        for h in range(s.hq):
            worst[r0:r1, h] = (amp[r0:r1, h] @ k[h // G].T).max(1) / s.d ** 0.5
    err = np.abs(f64(lse) - ref_lse)[has]
    bound = (half + 2.0 ** -20) * worst[has] + (2.0 ** -8 if blocks else 0) + 2.0 ** -20
    say(f"lse error {err.max():.2e}, of its bound {(err / bound).max():.2f}")
    assert (err <= bound).all()


@pytest.mark.parametrize("store", ["bf16", "i8"])
@pytest.mark.parametrize("hq,d", [(8, 128), (8, 64), (48, 128)])
def test_single_tokens_are_rounded_once(hq, d, store):
    """A single token's output is its own rounding, 2^-8, away from fp32's: queries and
    probabilities are within 2^-16.  A score is so off by at most 2^-16 of its products' magnitudes
    (and 2^-20 for fp32), a weight by twice the largest such error and 2^-16, and so the output by
    that of its weights' sum of magnitudes of values."""
    s = Scene(store, [1, 1, 1], [2, 20, 90], hq=hq, hkv=2, d=d, seed=37)
    out = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out)
    torch.cuda.synchronize()
    kp, vp = s.pages64()
    q, G, got = f64(s.q), s.hq // s.hkv, f64(out)
    most = 0.0
    for b in range(s.B):
        n = int(s.kv_len[b])
        ids = s.table[b][:-(-n // s.page)]
        k = np.concatenate([kp[i] for i in ids], 1)[:, :n]
        v = np.concatenate([vp[i] for i in ids], 2)[:, :, :n]
        for h in range(s.hq):
            x = k[h // G] @ q[b, h] / s.d ** 0.5
            off = (np.abs(k[h // G]) @ np.abs(q[b, h])).max() / s.d ** 0.5 * (2.0 ** -16 + 2.0 ** -20)
            p = np.exp(x - x.max())
            p /= p.sum()
            ref, mag = v[h // G] @ p, np.abs(v[h // G]) @ p
            bound = 2.0 ** -8 * np.abs(ref) + (2 * off + 2.0 ** -16 + 2.0 ** -20) * mag
            err = np.abs(got[b, h] - ref)
            most = max(most, float((err / bound).max()))
            assert (err <= bound).all(), (b, h, most)
    say(f"single tokens {store}: at most {most:.2f} of the bound")


@pytest.mark.parametrize("store", STORES)
def test_prime_groups_and_many_requests(store):
    """37 query heads a kv-head (no divisor up to 32), and 300 requests, some of them empty."""
    for kw in (dict(n=[1, 1], ctx=[70, 500], hq=37, hkv=1, d=64),
               dict(n=[(3 * i) % 4 for i in range(300)], ctx=[i % 90 for i in range(300)], hq=2,
                    hkv=1, d=64)):
        s = Scene(store, seed=31, **kw)
        out, lse = s.out(), s.lse()
        c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(max_chunk=max(s.n)), s.q, out, s.pos, lse)
        torch.cuda.synchronize()
        check_attend(s, out, lse, *dense64(s, s.q, s.pos.cpu().numpy()))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("hq,d", [(33, 128), (40, 128), (64, 64), (66, 64), (130, 128)])
def test_single_tokens_of_more_heads_than_a_unit(hq, d, store):
    """Over 32 query heads a kv-head: int8 in two parts of them, where they are even and up to
    64, and blocks of rows otherwise."""
    s = Scene(store, [1, 1, 1], [70, 900, 0], hq=2 * hq, hkv=2, d=d, seed=34)
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(max_chunk=1), s.q, out, s.pos, lse)
    torch.cuda.synchronize()
    check_attend(s, out, lse, *dense64(s, s.q, s.pos.cpu().numpy()))


def test_offsets_past_32_bits():
    """A cache whose later pages lie beyond 2^32 elements from its start (4.4 GB each of keys
    and values, int8): written, read back and attended there."""
    hkv, d, page = 8, 128, 256
    n_pages = (1 << 32) // (hkv * d * page) + 40
    s = Scene("i8", [1, 90], [400, 130], hq=16, hkv=hkv, page=page, seed=33)
    big = [torch.zeros((n_pages, hkv, *x), dtype=torch.int8, device="cuda")
           for x in ((page, d), (d, page))]
    scales = [torch.ones((n_pages, hkv, page), device="cuda") for _ in range(2)]
    used = s.table >= 0
    far = s.table.copy()
    far[used] = n_pages - 1 - s.table[used]
    for b in range(s.B):
        for c in range(s.max_pages):
            if s.table[b, c] >= 0:
                for dst, src in zip((*big, *scales), (s.kp, s.vp, s.ks, s.vs)):
                    dst[far[b, c]] = src[s.table[b, c]]
    cache = c2kv.Cache(*big, *scales)
    outs = []
    for c, t in ((s.cache, s.table), (cache, far)):
        ch = s.chunks(table=t)
        c2kv.c2kv_cache_write(s.cfg, c, ch, s.k, s.v, s.pos)
        k, v, o = torch.empty_like(s.k), torch.empty_like(s.v), s.out()
        c2kv.c2kv_cache_read(s.cfg, c, ch, k, v)
        c2kv.c2kv_cache_attend(s.cfg, c, ch, s.q, o, s.pos)
        outs.append((k, v, o))
    torch.cuda.synchronize()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("shape", [dict(n=[1, 1, 1, 1, 1], ctx=[10, 200, 300, 64, 30]),
                                   dict(n=[5, 90, 2, 40, 3], ctx=[10, 200, 300, 64, 30])])
def test_attend_missing_pages_and_lengths(shape, store):
    """Pages that are not there hide their keys, chunks longer than their cache give rows
    without keys, lengths past the block table stop at its end: all as the oracle says.
    (The index rules are checked on the CPU for any contents.)"""
    s = Scene(store, seed=5, hq=8, hkv=2, **shape)
    say(f"attend with missing pages {store} {shape}")
    s.table[1, 1] = -1                       # a hole in the middle
    s.table[2, 0] = s.n_pages + 3            # a number past the supply
    s.table[3, :] = -5                       # nothing at all
    s.kv_len[4] = s.n[4] - 1                 # the first row sees nothing
    s.kv_len[0] = s.max_pages * s.page + 70  # longer than the block-table row names
    s.table[0, 1] = s.table[1, 0]            # shared with another request
    kp, vp = s.pages64()
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out, s.pos, lse)
    torch.cuda.synchronize()
    ref = cache_oracle.attend(f64(s.q), s.pos.cpu().numpy(), kp, vp, s.tok_off, s.kv_len,
                              s.table, s.base)
    check_attend(s, out, lse, *ref)


@pytest.mark.parametrize("store", STORES)
def test_write_skips_missing_pages_of_long_chunks(store):
    s = Scene(store, [700, 3, 500], [10, 0, 5], seed=9)
    s.table[0, 1] = -1
    s.table[2, 0] = s.n_pages
    s.kv_len[1] = 1
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    rows = np.array([r for r in sorted(where) if where[r][2] is not None])
    for t in (s.kp, s.vp):
        t.zero_()
    c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(), s.k, s.v)
    torch.cuda.synchronize()
    assert (f64(s.kp) != 0).any((1, 3)).sum() == len(rows)
    assert (f64(s.vp) != 0).any((1, 2)).sum() == len(rows)
    page = np.array([where[r][2] for r in rows])
    at = np.array([where[r][3] for r in rows])
    kp, vp = s.pages64()
    tol = dict(f32=0, bf16=0, i8=0.03)[store]
    assert np.abs(kp[page, :, at] - f64(s.k)[rows]).max() <= tol
    assert np.abs(vp[page, :, :, at] - f64(s.v)[rows]).max() <= tol


@pytest.mark.parametrize("store", STORES)
def test_write_and_read_skip_missing_pages(store):
    s = Scene(store, [70, 3, 90], [10, 0, 5], seed=9)
    s.table[0, 1] = -1
    s.table[2, 0] = s.n_pages
    s.kv_len[1] = 1                          # the first two tokens have no place
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    rows = np.array([r for r in sorted(where) if where[r][2] is not None])
    for hint in (1, 100):
        for t in (s.kp, s.vp):
            t.zero_()
        c2kv.c2kv_cache_write(s.cfg, s.cache, s.chunks(max_chunk=hint), s.k, s.v)
        torch.cuda.synchronize()
        written = (f64(s.kp) != 0).any((1, 3)).sum()
        assert written == len(rows), (written, len(rows))
        k, v = (torch.full((s.n_tokens, s.hkv, s.d), 7.0, dtype=s.act, device="cuda")
                for _ in range(2))
        c2kv.c2kv_cache_read(s.cfg, s.cache, s.chunks(), k, v)
        torch.cuda.synchronize()
        rest = np.setdiff1d(np.arange(s.n_tokens), rows)
        assert (k[rest] == 7).all() and (v[rest] == 7).all()
        tol = dict(f32=0, bf16=0, i8=0.03)[store]
        assert (k[rows].float() - s.k[rows].float()).abs().max() <= tol
        assert (v[rows].float() - s.v[rows].float()).abs().max() <= tol


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("n", [[1, 1], [4, 3], [70, 100]])
def test_attend_ignores_what_lies_behind(n, store):
    """NaN and infinity behind the last cached token, and in pages that belong to nobody."""
    s = Scene(store, n, [20, 100], seed=11)
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out, s.pos, lse)
    used = torch.zeros((s.n_pages, s.page), dtype=torch.bool)
    for b in range(s.B):
        for j in range(int(s.kv_len[b])):
            used[s.table[b, j // s.page], j % s.page] = True
    bad = ~used.cuda()
    for x in (float("nan"), float("inf")):
        if store == "i8":
            s.ks.masked_fill_(bad[:, None], x)
            s.vs.masked_fill_(bad[:, None], -x)
        else:
            s.kp.masked_fill_(bad[:, None, :, None], x)
            s.vp.masked_fill_(bad[:, None, None, :], -x)
        out2, lse2 = s.out(), s.lse()
        c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out2, s.pos, lse2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_attend_nan_query_stays_in_its_row():
    s = Scene("bf16", [3, 40], [200, 30], seed=12)
    out = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out, s.pos)
    q = s.q.clone()
    q[1, 3] = float("nan")
    q[20, 0] = float("nan")
    out2 = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), q, out2, s.pos)
    torch.cuda.synchronize()
    assert torch.isnan(out2[1, 3]).all() and torch.isnan(out2[20, 0]).all()
    out2[1, 3], out2[20, 0] = out[1, 3], out[20, 0]
    assert torch.isfinite(out2).all()


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("n,hq", [([5, 3], 8), ([40, 90], 8), ([300, 70], 2), ([9, 2], 24)])
def test_attend_values_that_later_tokens_see(n, hq, store):
    """Infinities and NaN in the values (and keys) of a chunk's own tokens reach the tokens
    that see them, column by column, and no token before them."""
    s = Scene(store, n, [70, 130], hq=hq, hkv=2, seed=21)
    say(f"values not finite {store} {n}")
    out = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out, s.pos)
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    inf, nan = float("inf"), float("nan")
    want = out.clone().float()
    G = hq // s.hkv
    for b, (t, h, d, x) in enumerate([(n[0] // 2, 0, 7, inf), (n[1] - 1, 1, 100, nan)]):
        r0, r1 = int(s.tok_off[b]), int(s.tok_off[b + 1])
        _, _, page, at = where[r0 + t]
        heads = slice(h * G, (h + 1) * G)
        if store == "i8":
            s.vs[page, h, at] = nan
            want[r0 + t:r1, heads] = nan
        else:
            s.vp[page, h, d, at] = x
            want[r0 + t:r1, heads, d] = x
            if b == 0:                       # and one of each sign in another column
                s.vp[page, h, d + 1, at] = -inf
                want[r0 + t:r1, heads, d + 1] = -inf
                s.vp[where[r0 + t + 1][2], h, d + 1, where[r0 + t + 1][3]] = inf
                want[r0 + t + 1:r1, heads, d + 1] = nan
    out2 = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out2, s.pos)
    torch.cuda.synchronize()
    got = out2.float()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[fine], want[fine])
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])


@pytest.mark.parametrize("store", ["f32", "bf16"])
@pytest.mark.parametrize("n,hq,hint", [
    ([1, 1], 8, 1), ([1, 1], 48, 1),             # single tokens, up to 16 and up to 32 heads
    ([5, 3], 8, 1), ([5, 3], 8, 5), ([5, 3], 8, 10_000),      # a chunk by rows and by blocks
    ([40, 90], 8, 90), ([300, 70], 2, 300),
])
def test_attend_keys_that_are_not_finite(n, hq, hint, store):
    """Infinities and NaN in visible keys, whatever the kernel: a score of -inf is a key without
    weight, one of +inf or NaN makes its row NaN, and rows and heads that do not see the key
    are as they were.  The row's own sign of the query decides which."""
    s = Scene(store, n, [70, 130], hq=hq, hkv=2, seed=22)
    say(f"keys not finite {store} {n} hint {hint}")
    inf = float("inf")
    G = hq // s.hkv
    # query values whose products with the odd keys have a sign, single-number ones among them
    q = s.q
    q[:, :, 7] = torch.where(q[:, :, 7] < 0, -0.5, 0.5)
    q[:, :, 9] = torch.where(q[:, :, 9] < 0, -1.25, 0.75)
    ch = s.chunks(max_chunk=hint)
    was = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, q, was)
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    _, _, page, at = where[int(s.tok_off[0]) + n[0] // 2]
    s.kp[page, 0, at, 7] = inf
    _, _, page, at = where[int(s.tok_off[1]) + n[1] - 1]
    s.kp[page, 0, at, 9], s.kp[page, 0, at, 7] = -inf, inf
    s.kp[page, 1, at, 100] = float("nan")
    s.kp[s.table[1, 0], 1, 17, 9] = -inf         # in the context, seen by all
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, q, out, None, lse)
    torch.cuda.synchronize()
    ref, ref_lse, has = dense64(s, q, None)
    assert has.all()
    nan = np.isnan(ref)
    assert nan.any() and not nan.all() and (nan.all(-1) == nan.any(-1)).all()
    got = f64(out)
    assert (np.isnan(got) == nan).all()
    assert (np.isnan(f64(lse)) == nan.any(-1)).all()
    fine = ~nan.any(-1)
    err, lerr = np.abs(got - ref)[fine], np.abs(f64(lse) - ref_lse)[fine]
    if store == "f32":
        assert err.max() <= 1e-5 and lerr.max() <= 1e-5
    else:
        assert err.max() <= 2e-2 and err.mean() <= 1e-2 and lerr.max() <= 5e-2
    before = int(s.tok_off[0]) + n[0] // 2       # the first request's tokens that do not see it
    assert torch.equal(out[:before], was[:before])
    assert torch.equal(out[:n[0], G:], was[:n[0], G:])


@pytest.mark.parametrize("n,hq,hint", [([1, 1], 8, 1), ([1, 1], 80, 1), ([5, 3], 8, 5),
                                       ([90, 40], 8, 90)])
def test_attend_int8_key_scales_that_are_nan(n, hq, hint):
    """The scale of a cached key that held an infinity or a NaN: rows that see it are NaN, and
    no others."""
    s = Scene("i8", n, [70, 130], hq=hq, hkv=2, seed=24)
    say(f"key scales not finite {n} {hq}")
    G, t = hq // 2, n[0] // 2
    ch = s.chunks(max_chunk=hint)
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, s.q, out, s.pos, lse)
    where = cache_oracle.places(s.tok_off, s.kv_len, s.table, s.page, s.n_pages, s.n_tokens)
    s.ks[where[t][2], 1, where[t][3]] = float("nan")
    out2, lse2 = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, s.q, out2, s.pos, lse2)
    torch.cuda.synchronize()
    assert torch.isnan(out2[t:n[0], G:]).all() and torch.isnan(lse2[t:n[0], G:]).all()
    out2[t:n[0], G:], lse2[t:n[0], G:] = out[t:n[0], G:], lse[t:n[0], G:]
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("hq", [8, 48])
def test_single_tokens_see_values_that_are_not_finite(hq, store):
    """An infinite value makes its column infinite, whatever the weights, a NaN makes it NaN."""
    s = Scene(store, [1, 1], [70, 130], hq=hq, hkv=2, seed=25)
    ch, G, inf = s.chunks(), hq // 2, float("inf")
    out = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, s.q, out, s.pos)
    want = out.clone()
    page = s.table[0, 0]
    if store == "i8":
        s.vs[page, 1, 9] = float("nan")
        want[0, G:] = float("nan")
    else:
        s.vp[page, 0, 3, 5], s.vp[page, 0, 4, 6], s.vp[page, 1, 7, 9] = inf, -inf, float("nan")
        want[0, :G, 3], want[0, :G, 4], want[0, G:, 7] = inf, -inf, float("nan")
    out2 = s.out()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, s.q, out2, s.pos)
    torch.cuda.synchronize()
    assert torch.equal(torch.isnan(out2), torch.isnan(want))
    assert torch.equal(out2.nan_to_num(0, inf, -inf), want.nan_to_num(0, inf, -inf))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("n,hint", [([1, 1], 1), ([5, 3], 5), ([100, 40], 100)])
def test_attend_infinite_queries(n, hint, store):
    """A query whose every score is -inf sees no key; one with a score of +inf is NaN."""
    s = Scene(store, n, [70, 130], seed=23)
    s.kp[..., 7] = -s.kp[..., 7].abs().clamp_min(1)
    s.q[0, 1, 7], s.q[n[0], 2, 7] = float("inf"), float("-inf")
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(max_chunk=hint), s.q, out, None, lse)
    torch.cuda.synchronize()
    assert (out[0, 1] == 0).all() and lse[0, 1] == float("-inf")
    assert torch.isnan(out[n[0], 2]).all() and torch.isnan(lse[n[0], 2])
    out[0, 1], out[n[0], 2] = 1, 1
    assert torch.isfinite(out).all() and (~torch.isfinite(lse)).sum() == 2


def test_attend_large_scores():
    """Scores of some hundreds: one key takes all, no overflow."""
    s = Scene("bf16", [1, 50], [300, 200], seed=13)
    q = s.q * 60
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), q, out, s.pos, lse)
    torch.cuda.synchronize()
    ref, ref_lse, _ = dense64(s, q, s.pos.cpu().numpy())
    # scores near 500 are off by up to 2^-8 of |q||k| / sqrt(d) ~ 60 * 11: 2.6 where two keys
    # compete, so only the lse (which moves no more than the scores) is compared
    assert torch.isfinite(out.float()).all()
    assert np.abs(f64(lse) - ref_lse).max() <= 60 * 11 * 2.0 ** -8


@pytest.mark.parametrize("store", STORES)
def test_softmax_scale_and_unturned_queries(store):
    s = Scene(store, [1, 37], [90, 200], seed=14)
    s.cfg.softmax_scale = 0.5 * s.d ** -0.5
    out, lse = s.out(), s.lse()
    c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, out, None, lse)
    torch.cuda.synchronize()
    check_attend(s, out, lse, *dense64(s, s.q / 2, None))


# ---- steps, streams, graphs -------------------------------------------------------

@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("n", [1, 20])
def test_graph_replays_follow_growing_lengths(store, n):
    """A captured step (write, attend, read back) replayed while lengths, offsets, positions
    and inputs change on the device, with eager work of the same kind between the replays."""
    s = Scene(store, [n, n, n], [40, 300, 0], seed=15, hq=8, hkv=2)
    spare = np.setdiff1d(np.arange(s.n_pages), s.table)
    grow = np.full((s.B, s.max_pages + 2), -1, np.int32)
    grow[:, :s.max_pages] = s.table
    pages = list(spare)
    s.table = grow
    ch = s.chunks(max_chunk=n)
    tok_off, kv_len, table = ch.tensors
    q, k, v, pos = (t.clone() for t in (s.q, s.k, s.v, s.pos))
    out, lse = s.out(), s.lse()
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    ws = c2kv.cache_attend_workspace(s.cfg, s.cache, ch)

    def step(out, lse, rk, rv, ws):
        c2kv.c2kv_cache_write(s.cfg, s.cache, ch, k, v, pos)
        c2kv.c2kv_cache_attend(s.cfg, s.cache, ch, q, out, pos, lse, workspace=ws)
        c2kv.c2kv_cache_read(s.cfg, s.cache, ch, rk, rv)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, lse, rk, rv, ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, lse, rk, rv, ws)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for i in range(5):
        kv_len += torch.tensor([1, 0, 2], dtype=torch.int32, device="cuda")
        for b in range(s.B):
            col = (int(kv_len[b]) - 1) // s.page
            if int(table[b, col]) < 0 and pages:
                table[b, col] = pages.pop()
        pos += 2
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        for t in (out, lse, rk, rv):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, rk, rv)]
        ref = [torch.empty_like(t) for t in got]
        step(*ref, c2kv.cache_attend_workspace(s.cfg, s.cache, ch))
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            assert torch.equal(a, b), f"replay {i}"


def test_two_streams_with_workspaces_of_their_own():
    a, b = Scene("bf16", [1, 5], [3000, 700], seed=16), Scene("i8", [300], [900], seed=17)
    ref, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in (a, b):
        o = s.out()
        c2kv.c2kv_cache_attend(s.cfg, s.cache, s.chunks(), s.q, o, s.pos)
        ref.append(o)
    chunks = [s.chunks() for s in (a, b)]
    ws = [c2kv.cache_attend_workspace(s.cfg, s.cache, c) for s, c in zip((a, b), chunks)]
    outs = [s.out() for s in (a, b)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, c, w, o, st in zip((a, b), chunks, ws, outs, streams):
            c2kv.c2kv_cache_attend(s.cfg, s.cache, c, s.q, o, s.pos, workspace=w, stream=st)
    torch.cuda.synchronize()
    for o, r in zip(outs, ref):
        assert torch.equal(o, r)


# ---- together ---------------------------------------------------------------------

@pytest.mark.parametrize("store", STORES)
def test_compose_then_grow(store):
    """A request's whole life: chunks stored in the pool by c2kv_pool_write, composed into
    pages, the prompt written behind them and attended in two chunks (as c2kv_compose_attend
    attends it at once), then single tokens; read back at the end."""
    say(f"compose then grow {store}")
    pool_dtype = store
    w = synth.small(pool_dtype=pool_dtype, batch=2, n_q_heads=8, n_kv_heads=2, suffix_len=37)
    dev = Dev(w)
    act = ACT[store]
    cfg = c2kv.attn_cfg(w.n_q_heads, w.n_kv_heads, w.head_dim, w.act_dtype, w.rope_base)
    # the pool's rows, stored from rows in the act dtype (keys as they are)
    rk, rv = dev.k.clone(), dev.v.clone()
    if store == "i8":
        rk = (dev.k.float() * dev.ks[..., None]).to(act)
        rv = (dev.v.float() * dev.vs[..., None]).to(act)
    pk, pv = torch.zeros_like(dev.k), torch.zeros_like(dev.v)
    ks = vs = None
    if store == "i8":
        ks, vs = torch.zeros_like(dev.ks), torch.zeros_like(dev.vs)
    pool = c2kv.pool_desc(pk, pv, ks, vs)
    c2kv.c2kv_pool_write(cfg, pool, torch.arange(len(pk), device="cuda"), rk, rv)
    plan = c2kv.Plan.for_workload(w).upload()
    B, S, Hq, D = dev.q.shape
    H, PS = w.n_kv_heads, plan.info["page_size"]
    ref, ref_lse = dev.out_like(), dev.lse_like()
    c2kv.c2kv_compose_attend(plan, pool, dev.q, dev.k_suf, dev.v_suf, ref, ref_lse)

    # pages for the composition and for what follows; int8 caches are written from rows
    n0, span = plan.requests()
    n_pages = plan.info["n_pages"] + 2 * B
    cols = -(-int(n0.max() + S + 4) // PS)
    table = np.full((B, cols), -1, np.int32)
    bt = plan.block_table()
    table[:, :bt.shape[1]] = bt
    free = list(range(plan.info["n_pages"], n_pages))
    for b in range(B):
        for c in range(-(-int(n0[b] + S + 4) // PS)):
            if table[b, c] < 0:
                table[b, c] = free.pop(0)
    kp = torch.full((n_pages, H, PS, D), float("nan"), dtype=act, device="cuda")
    vp = torch.full((n_pages, H, D, PS), float("nan"), dtype=act, device="cuda")
    c2kv.c2kv_compose(plan, pool, kp, vp)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()
    tab = i32(table)
    cache = c2kv.Cache(kp, vp)
    if store == "i8":
        all_off = i32(np.concatenate([[0], np.cumsum(n0)]))
        whole = c2kv.Chunks(all_off, i32(n0), tab, int(n0.sum()))
        ck, cv = (torch.empty((int(n0.sum()), H, D), dtype=act, device="cuda") for _ in range(2))
        c2kv.c2kv_cache_read(cfg, cache, whole, ck, cv)
        k8 = torch.zeros((n_pages, H, PS, D), dtype=torch.int8, device="cuda")
        v8 = torch.zeros((n_pages, H, D, PS), dtype=torch.int8, device="cuda")
        s8 = [torch.full((n_pages, H, PS), float("nan"), device="cuda") for _ in range(2)]
        cache = c2kv.Cache(k8, v8, *s8)
        c2kv.c2kv_cache_write(cfg, cache, whole, ck, cv)

    got = torch.empty_like(ref)
    done = 0
    for part in (20, S - 20 - 3, 1, 1, 1):       # a prompt in two chunks, then single tokens
        off = i32(np.arange(B + 1) * part)
        ch = c2kv.Chunks(off, i32(n0 + done + part), tab, B * part, max_chunk=part)
        take = lambda t: t[:, done:done + part].reshape(B * part, -1, D).contiguous()
        pos = i32(np.concatenate([span[b] + done + np.arange(part) for b in range(B)]))
        c2kv.c2kv_cache_write(cfg, cache, ch, take(dev.k_suf), take(dev.v_suf), pos)
        o = torch.empty((B * part, Hq, D), dtype=act, device="cuda")
        c2kv.c2kv_cache_attend(cfg, cache, ch, take(dev.q), o, pos)
        got[:, done:done + part] = o.reshape(B, part, Hq, D)
        done += part
    torch.cuda.synchronize()
    assert done == S
    err = (got.double() - ref.double()).abs()
    say(f"grown against composed: max {err.max():.2e}")
    # both are within the parity bar of the same sum; an int8 cache adds, for each key and
    # value, half a code: a scale of 4.5 / 127 at most for these values gives 0.018
    assert err.max() <= dict(f32=2e-5, bf16=4e-2, i8=6e-2)[store]

    # the suffix comes back, turned to its positions or back to where it came from
    ch = c2kv.Chunks(i32(np.arange(B + 1) * S), i32(n0 + S), tab, B * S)
    bk, bv = (torch.empty((B * S, H, D), dtype=act, device="cuda") for _ in range(2))
    pos = i32(np.concatenate([span[b] + np.arange(S) for b in range(B)]))
    c2kv.c2kv_cache_read(cfg, cache, ch, bk, bv, -pos)
    torch.cuda.synchronize()
    tol = dict(f32=2e-6, bf16=2.0 ** -7, i8=0.03)[store]
    assert (bv.float() - dev.v_suf.reshape(B * S, H, D).float()).abs().max() <= \
        (0 if store != "i8" else tol)
    # two roundings of the pair's values, or half a code and two roundings
    amp = dev.k_suf.float().abs().max().item()
    assert (bk.float() - dev.k_suf.reshape(B * S, H, D).float()).abs().max() <= tol * 2 * amp
