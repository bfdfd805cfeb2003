"""GPU parity of the decoder operators (root-mean-square norm, cache in 4 bits, attention over it, eviction) with their definitions
in 64-bit integers, bit for bit: everything is integer arithmetic, so no difference is allowed anywhere."""
import numpy as np
import pytest
import torch

from ivit_inputs import ExpParams, Scale
from ivit_inputs.gen import dyadic, scale_channels
from oracle import api as O
from oracle import decoder as D

pytestmark = pytest.mark.gpu


def _g():
    import gpu_util
    return gpu_util


def rand_i8(rng, shape, std=32):
    return np.clip(np.rint(rng.standard_normal(shape) * std), -128, 127).astype(np.int8)


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- root-mean-square norm ----

def norm_case(rng, rows, C, x32, h32, kind):
    """x, res, x ratio: ordinary, zeros in some rows, or the extremes of the types."""
    x = rng.standard_normal((rows, C)) * (20000 if x32 else 32)
    res = rng.standard_normal((rows, C)) * (3000 if h32 else 20)
    x, res = np.rint(x), np.rint(res)
    if kind == "extreme":
        x = rng.choice([-2.0 ** 31, 2.0 ** 31 - 1, 0, 1, -1] if x32 else [-128, 127, 0, -1], (rows, C))
        res = rng.choice([-2.0 ** 31, 2.0 ** 31 - 1, 2.0 ** 20, -2.0 ** 20, 0] if h32 else [-128, 127, 0], (rows, C))
    elif kind == "sparse":
        keep = rng.random((rows, C)) < 1.5 / C
        x, res = np.where(keep, x, 0), np.where(keep, res, 0)
        x[0], res[0] = 0, 0
    x = x.astype(np.int32) if x32 else np.clip(x, -128, 127).astype(np.int8)
    return x, res.astype(np.int32) if h32 else np.clip(res, -128, 127).astype(np.int8)


@pytest.mark.parametrize("kind", ["ordinary", "sparse", "extreme"])
@pytest.mark.parametrize("x32,h32", [(0, None), (1, None), (0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,C", [(1, 4), (1, 768), (3, 772), (130, 64), (197, 192), (700, 132), (40, 1000), (64, 4096), (2000, 2048), (9, 16384),
                                    (400, 5000)])
def test_rmsnorm_parity(rows, C, x32, h32, kind):
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(rows * 31 + C + 7 * x32 + 3 * (h32 or 0) + len(kind))
    x, res = norm_case(rng, rows, C, x32, h32 or 0, kind)
    xs = scale_channels(rng.uniform(0.5, 1.5, C) * ((500.0 if h32 else 10.0) / (20000.0 if x32 else 1100.0)))
    rs = Scale(*dyadic(0.96875))
    for dynamic, M_ln, ratio in ((False, 20, 32.0 * np.sqrt(C) / 2 ** 20), (True, 22, 0.4), (True, 8, 0.9)):
        gs = scale_channels(rng.uniform(0.8, 1.1, C) * min(ratio, 0.9))
        want, top, total = D.rmsnorm(x, (gs.mult, gs.shift), M_ln, (xs.mult, xs.shift), None if h32 is None else res, (rs.mult, rs.shift), h32 == 1,
                                     dynamic)
        dx, dr = g.dev(x), None if h32 is None else g.dev(res)
        sums = None if h32 is None else g.dev(np.zeros_like(res))
        rm = torch.zeros(rows, dtype=torch.int32, device="cuda") if dynamic else None
        got = c.rmsnorm(dx, g.binding.DevScale(gs, "cuda"), x_scale=g.binding.DevScale(xs, "cuda"), res=dr,
                        res_scale=None if h32 is None else g.binding.DevScale(rs, "cuda"), M_ln=M_ln, sum_out=sums, row_max=rm)
        what = f"M_ln {M_ln} dynamic {dynamic}"
        g.assert_equal(g.host(got), want.astype(np.int8), what)
        if dynamic:
            g.assert_equal(g.host(rm), top.astype(np.int32), what + " row_max")
        if h32 is not None:
            g.assert_equal(g.host(sums), total.astype(sums.cpu().numpy().dtype), what + " sum")
            # the stream in place, without and with the sum wanted
            got = c.rmsnorm(dx, g.binding.DevScale(gs, "cuda"), x_scale=g.binding.DevScale(xs, "cuda"), res=dr,
                            res_scale=g.binding.DevScale(rs, "cuda"), M_ln=M_ln, row_max=rm)
            g.assert_equal(g.host(got), want.astype(np.int8), what + " no sum")
            c.rmsnorm(dx, g.binding.DevScale(gs, "cuda"), x_scale=g.binding.DevScale(xs, "cuda"), res=dr,
                      res_scale=g.binding.DevScale(rs, "cuda"), M_ln=M_ln, sum_out=dr, row_max=rm, out=got)
            g.assert_equal(g.host(got), want.astype(np.int8), what + " in place")
            g.assert_equal(g.host(dr), total.astype(res.dtype), what + " stream in place")
    assert c.poll_status() == 0


@pytest.mark.parametrize("shift", [31, 32, 33, 39, 40, 41, 54, 55, 61, 62])
@pytest.mark.parametrize("x32,h32", [(0, 0), (1, 1)])
def test_rmsnorm_every_shift(shift, x32, h32):
    """Per-tensor scales, and per-channel ones, over the whole range of shifts, at both ends of the multipliers."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(shift)
    rows, C = 37, 516
    x, res = norm_case(rng, rows, C, x32, h32, "extreme")
    for mult in (1, 2 ** 31 - 1):
        s = Scale(mult, shift)
        sc = Scale(np.full(C, mult, np.int32), np.full(C, shift, np.uint8))
        want, top, total = D.rmsnorm(x, (mult, shift), 21, (mult, shift), res, (mult, shift), h32 == 1, True)
        for per in (s, sc):
            sums, rm = g.dev(np.zeros_like(res)), torch.zeros(rows, dtype=torch.int32, device="cuda")
            got = c.rmsnorm(g.dev(x), g.binding.DevScale(per, "cuda"), x_scale=g.binding.DevScale(per, "cuda"), res=g.dev(res),
                            res_scale=g.binding.DevScale(s, "cuda"), M_ln=21, sum_out=sums, row_max=rm)
            g.assert_equal(g.host(got), want.astype(np.int8), f"mult {mult}")
            g.assert_equal(g.host(rm), top.astype(np.int32), f"mult {mult} row_max")
            g.assert_equal(g.host(sums), total.astype(res.dtype), f"mult {mult} sum")


def test_rmsnorm_leaves_the_rest_alone():
    """Columns past C of every tensor, and rows past the last, keep what they held."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(3)
    for rows, C, ld in ((5, 100, 112), (2, 772, 1024), (1, 4, 16), (300, 36, 48)):
        x, res = norm_case(rng, rows, C, 0, 0, "ordinary")
        bx = torch.full((rows + 1, ld), 77, dtype=torch.int8, device="cuda")
        br, bo = bx.clone(), bx.clone()
        bx[:rows, :C], br[:rows, :C] = cuda(x), cuda(res)
        s = g.binding.DevScale(Scale(*dyadic(0.01)), "cuda")
        c.rmsnorm(bx[:rows, :C], s, x_scale=s, res=br[:rows, :C], res_scale=s, sum_out=br[:rows, :C], out=bo[:rows, :C])
        for t in (bx, br, bo):
            assert (t[rows:] == 77).all() and (t[:, C:] == 77).all()


# ---- cache in 4 bits: append ----

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
@pytest.mark.parametrize("heads,tokens", [(1, 1), (3, 29), (8, 200), (5, 1500)])
def test_append_parity(d, page, heads, tokens):
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(d + page + heads + tokens)
    pages = -(-tokens // page) + 2
    k, v = rand_i8(rng, (tokens, heads * d)), rand_i8(rng, (tokens, heads * d), 50)
    k[rng.random(k.shape) < 0.01] = -128
    k[0, :32], v[-1, :d] = 0, 0                                   # groups of zeros
    v[0, :d] = np.where(np.arange(d) == 5, 1, 0)
    qkv = np.concatenate([np.full((tokens, 32), 99, np.int8), k, v], 1)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    if tokens > 10:
        slots[[3, 7]] = -1, -2 ** 40
    ref = D.Cache(pages, heads, d, page)
    before = rng.integers(0, 256, (pages, heads, page * (d + d // 32 + 1))).astype(np.uint8)
    ref = D.Cache.of_bytes(before, d, page)
    ref.append(k, v, slots)
    cache = g.binding.Kv4Cache(cuda(before), d, page)
    dq = g.dev(qkv)
    c.kv4_append(cache, dq[:, 32:32 + heads * d], dq[:, 32 + heads * d:32 + 2 * heads * d], cuda(slots))
    g.assert_equal(g.host(cache.pool), ref.to_bytes(), "pool")
    assert c.poll_status() == 0
    # a slot past the pool is left out and reported; a call without tokens does nothing
    slots[0] = pages * page
    c.kv4_append(cache, dq[:1, 32:32 + heads * d], dq[:1, 32 + heads * d:32 + 2 * heads * d], cuda(slots[:1]))
    torch.cuda.synchronize()
    assert c.poll_status() == -3 and c.poll_status() == 0
    g.assert_equal(g.host(cache.pool), ref.to_bytes(), "pool after a bad slot")
    c.kv4_append(cache, dq[:0, 32:32 + heads * d], dq[:0, 32 + heads * d:32 + 2 * heads * d], cuda(slots[:0]))


def test_append_every_value():
    """Every int8 value against every step a group can have."""
    g, c = _g(), _g().ctx()
    top = np.repeat(np.arange(129), 256)                          # largest magnitude of the group
    x = np.tile(np.arange(-128, 128), 129)
    use = np.abs(x) <= top
    top, x = top[use], x[use]
    tokens, d = len(x), 64
    k, v = np.zeros((tokens, d), np.int64), np.zeros((tokens, d), np.int64)
    k[:, 0], k[:, 17] = x, -top
    k[:, 40], k[:, 33] = x, -top
    v[:, 1], v[:, 63] = x, -top
    k, v = k.astype(np.int8), v.astype(np.int8)
    pages = -(-tokens // 256)
    ref = D.Cache(pages, 1, d, 256)
    slots = np.arange(tokens, dtype=np.int64)
    ref.append(k, v, slots)
    cache = g.binding.Kv4Cache.empty(pages, 1, d, 256, "cuda")
    cache.pool.fill_(0x88)
    cache.pool.view(pages, -1)[:, :] = cuda(D.Cache(pages, 1, d, 256).to_bytes()).view(pages, -1)
    c.kv4_append(cache, cuda(k), cuda(v), cuda(slots))
    g.assert_equal(g.host(cache.pool), ref.to_bytes(), "pool")


# ---- attention over it ----

def filled(rng, pages, heads, d, page, std=24):
    ref = D.Cache(pages, heads, d, page)
    ref.ks = rng.integers(0, 148, ref.ks.shape) // rng.integers(1, 9, ref.ks.shape)
    ref.vs = rng.integers(0, 148, ref.vs.shape) // rng.integers(1, 9, ref.vs.shape)
    ref.kc, ref.vc = rng.integers(-7, 8, ref.kc.shape), rng.integers(-7, 8, ref.vc.shape)
    return ref


def attend(c, g, ref, q, heads_q, tq, lens, table, max_q=None, max_len=None, qk=None, pv=None, I0=17, N=15, weights=False, ldw=None, out=None):
    d, page, hk = ref.d, ref.page, ref.kc.shape[1]
    cache = g.binding.Kv4Cache(cuda(ref.to_bytes()), d, page)
    qs = np.concatenate([[0], np.cumsum(tq)]).astype(np.int32)
    qk = qk or dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40))
    pv = pv or dyadic(1 / 128)
    max_q = max(list(tq) + [0]) if max_q is None else max_q
    max_len = max(list(lens) + [0]) if max_len is None else max_len
    w0 = np.arange(len(lens) * hk * (ldw or table.shape[1] * page), dtype=np.int64).reshape(len(lens), hk, -1) if weights else None
    if out is None:
        out = np.full(q.shape, 55, np.int8)
    dout, dw = cuda(out), None if w0 is None else cuda(w0)
    c.kv4_attention(cache, cuda(q), cuda(qs), cuda(np.asarray(lens, np.int32)), cuda(np.asarray(table, np.int32)), g.binding.DevScale.of(*qk),
                    ExpParams(I0, N), g.binding.DevScale.of(*pv), max_q, max_len, out=dout, weights=dw)
    want, ww = D.attention(ref, q, heads_q, qs, lens, table, qk, I0, N, pv, out, w0)
    g.assert_equal(g.host(dout), want.astype(np.int8), "out")
    if weights:
        g.assert_equal(g.host(dw), ww, "weights")
    return g.host(dout)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 64, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (6, 6), (8, 4), (9, 3), (4, 1), (14, 2), (16, 2), (17, 1), (40, 2)])
def test_attention_decode(d, page, hq, hk):
    """One query token for each of sequences of 0, 1, ... keys; rows of no sequence stay; with and without weights."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(d + page + 17 * hq + hk)
    lens = [0, 1, 2, 31, 32, 33, 63, 64, 65, page - 1, page, page + 1, 300, 511, 700]
    B, np_ = len(lens), -(-max(lens) // page)
    ref = filled(rng, B * np_ + 3, hk, d, page)
    table = rng.permutation(B * np_ + 3)[:B * np_].reshape(B, np_)
    q = rand_i8(rng, (B + 3, hq * d))                              # three rows behind the last sequence
    for w in (False, True):
        got = attend(c, g, ref, q, hq, [1] * B, lens, table, weights=w)
        assert (got[B:] == 55).all()
    assert c.poll_status() == 0


@pytest.mark.parametrize("d,page,hq,hk", [(64, 32, 4, 4), (128, 64, 8, 2), (128, 32, 7, 1), (64, 128, 16, 1), (128, 256, 3, 3)])
def test_attention_query_rows(d, page, hq, hk):
    """Several query tokens per sequence: causal; fewer keys than queries, so that the first rows see nothing; no queries at all."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(d + page + hq)
    tq = [5, 0, 1, 33, 70, 9, 2, 17]
    lens = [5, 40, 1, 20, 70, 333, 0, 160]
    np_ = -(-max(lens) // page)
    ref = filled(rng, len(lens) * np_, hk, d, page)
    table = rng.permutation(len(lens) * np_).reshape(len(lens), np_)
    q = rand_i8(rng, (sum(tq), hq * d))
    attend(c, g, ref, q, hq, tq, lens, table)
    attend(c, g, ref, q, hq, tq, lens, table, weights=True)
    # the same launch sized for more than there is
    attend(c, g, ref, q, hq, tq, lens, table, max_q=90, max_len=np_ * page, weights=True, ldw=np_ * page + 5)
    assert c.poll_status() == 0


@pytest.mark.parametrize("I0,N", [(17, 15), (1, 14), (1, 23), (255, 15), (16384, 0), (32767, 9), (3, 22), (100, 8)])
def test_attention_exponentials(I0, N):
    """The corners of ShiftExp's constants, scores that saturate, equal scores, steps of zero."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(I0 + N)
    d, page, hk, hq = 128, 32, 2, 4
    lens = [257, 90, 1]
    ref = filled(rng, 3 * 9, hk, d, page)
    ref.ks[::5], ref.vs[::7] = 147, 147
    ref.kc[::3], ref.vc[::5] = 7, -7
    table = np.arange(27).reshape(3, 9)
    q = rng.choice([-128, 127, 0, 3], (3, hq * d)).astype(np.int8)
    for ratio in (2.0 ** -30, 2e-5, 1e-3, 0.99):
        attend(c, g, ref, q, hq, [1, 1, 1], lens, table, qk=dyadic(ratio), pv=dyadic(0.9), I0=I0, N=N, weights=True)
    ref.vs[:], ref.ks[:] = 0, 0
    attend(c, g, ref, q, hq, [1, 1, 1], lens, table, I0=I0, N=N, weights=True)


@pytest.mark.parametrize("d,page,hq,hk,L", [(64, 32, 1, 1, 3000), (128, 64, 4, 1, 9001), (128, 256, 16, 1, 20000), (64, 128, 8, 1, 40001), (128, 128, 17, 1, 5003)])
def test_attention_long_rows(d, page, hq, hk, L):
    """Rows long enough to be split, every key of equal weight at the end of the range of a code: the largest sums."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(L)
    np_ = -(-L // page)
    ref = filled(rng, np_, hk, d, page)
    table = rng.permutation(np_)[None]
    q = rand_i8(rng, (2, hq * d))
    attend(c, g, ref, q, hq, [2], [L], table, weights=True)
    ref.vc[:], ref.vs[:], ref.ks[:] = 7, 147, 0
    attend(c, g, ref, q, hq, [2], [L], table, weights=True, pv=dyadic(1 / 400))


@pytest.mark.parametrize("B,hk,G,d,L", [(1, 8, 4, 64, 11000), (2, 5, 1, 128, 12100), (3, 5, 2, 64, 9001), (4, 6, 3, 128, 6400), (11, 3, 5, 64, 4500),
                                        (15, 3, 8, 128, 3300), (37, 2, 4, 64, 2500), (1, 7, 2, 128, 30001), (1, 1, 7, 64, 33000)])
def test_attention_clusters(B, hk, G, d, L):
    """Clusters of every size, sequences that use all of their cluster, some of it, or one CTA of it, and none at all."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(B * 100 + hk)
    page = 64
    lens = [L] + [int(v) for v in rng.integers(0, L + 1, B - 1)]
    if B > 2:
        lens[1], lens[2] = 0, 33
    np_ = -(-L // page)
    pages = min(B * np_, 900)
    ref = filled(rng, pages, hk, d, page)
    table = rng.integers(0, pages, (B, np_))                      # (sequences may share pages)
    attend(c, g, ref, rand_i8(rng, (B, hk * G * d)), hk * G, [1] * B, lens, table, weights=True)
    attend(c, g, ref, rand_i8(rng, (B, hk * G * d)), hk * G, [1] * B, lens, table)
    assert c.poll_status() == 0


@pytest.mark.parametrize("B", [40, 128, 129])
def test_attention_uneven_batches(B):
    """Batches whose sequences are taken longest first (up to 128 of them), with equal lengths among them, and one too large for that."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(B)
    d, page, hk = 64, 32, 4
    lens = rng.integers(0, 1500, B)
    lens[::3] = 600
    lens[5] = 0
    np_ = 47
    ref = filled(rng, 400, hk, d, page)
    attend(c, g, ref, rand_i8(rng, (B, 2 * hk * d)), 2 * hk, [1] * B, lens, rng.integers(0, 400, (B, np_)), weights=True, max_len=1500)
    assert c.poll_status() == 0


@pytest.mark.parametrize("B,hk,G,L,tq", [(40, 4, 2, 4000, 1), (128, 2, 1, 2600, 1), (129, 2, 1, 2600, 1), (40, 2, 14, 300, 1), (40, 2, 9, 700, 1), (1, 2, 8, 13500, 76)])
def test_attention_forms(B, hk, G, L, tq):
    """Long uneven batches (16 warps a CTA, longest first), and CTAs of sixteen query rows: some of them never there, clusters of them."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(B + G)
    d, page = 64, 64
    lens = rng.integers(0, L + 1, B)
    lens[0], lens[-1] = L, L
    np_ = -(-L // page)
    ref = filled(rng, 250, hk, d, page)
    attend(c, g, ref, rand_i8(rng, (B * tq, G * hk * d)), G * hk, [tq] * B, lens, rng.integers(0, 250, (B, np_)), weights=True)
    attend(c, g, ref, rand_i8(rng, (B * tq, G * hk * d)), G * hk, [tq] * B, lens, rng.integers(0, 250, (B, np_)))
    assert c.poll_status() == 0


def test_attention_longest():
    """The longest sequence that the entry point takes."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(11)
    L, page = 196608, 256
    ref = filled(rng, L // page, 1, 64, page)
    ref.vc[:], ref.vs[:] = 7, 147
    attend(c, g, ref, rand_i8(rng, (1, 64 * 5)), 5, [1], [L], np.arange(L // page)[None], weights=True)
    assert c.poll_status() == 0


def test_attention_far_pages():
    """Pages more than 2^32 bytes into the pool."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(12)
    d, page, hk = 128, 256, 4
    block = page * (d + d // 32 + 1)
    pages = (5 << 30) // (hk * block)
    small = filled(rng, 6, hk, d, page)
    pool = torch.zeros((pages, hk, block), dtype=torch.uint8, device="cuda")
    at = [pages - 1, 0, pages - 3, pages // 2, pages - 2, pages // 2 + 7]
    pool[at] = cuda(small.to_bytes())
    cache = g.binding.Kv4Cache(pool, d, page)
    q = rand_i8(rng, (2, 8 * d))
    table, lens, qs = np.arange(6).reshape(2, 3), [700, 768], np.array([0, 1, 2])
    out = torch.zeros((2, 8 * d), dtype=torch.int8, device="cuda")
    qk, pv = dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40)), dyadic(1 / 128)
    far = cuda(np.array(at, np.int32)[table])
    c.kv4_attention(cache, cuda(q), cuda(qs.astype(np.int32)), cuda(np.array(lens, np.int32)), far, g.binding.DevScale.of(*qk), ExpParams(17, 15),
                    g.binding.DevScale.of(*pv), 1, 768, out=out)
    want, _ = D.attention(small, q, 8, qs, lens, table, qk, 17, 15, pv, np.zeros_like(q))
    g.assert_equal(g.host(out), want.astype(np.int8), "out")
    # a row appended there, and eviction that moves rows there
    k, v = rand_i8(rng, (1, hk * d)), rand_i8(rng, (1, hk * d))
    small.append(k, v, [2 * page + 200])
    c.kv4_append(cache, cuda(k), cuda(v), cuda(np.array([at[2] * page + 200])))
    w = rng.integers(0, 1 << 40, (2, hk, 768))
    kept, new = c.kv4_evict(cache, cuda(w), cuda(np.array(lens, np.int32)), far, 300, 4, 32, 768, weights_out=torch.empty((2, hk, 300), dtype=torch.int64, device="cuda"))
    wk, wn, _, bytes_ = D.evict(small, w, lens, table, table, 300, 300, 4, 32)
    g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
    g.assert_equal(g.host(pool[at]), bytes_, "pool")


def test_attention_indices_that_point_nowhere():
    """Pages outside the pool are not read: their keys are not seen, and the call says so.  The same for lengths past max_len,
    more queries than max_q, and rows past the end of Q."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(5)
    d, page, hk, hq = 64, 32, 2, 4
    lens, tq = [100, 64, 70], [1, 3, 1]
    ref = filled(rng, 12, hk, d, page)
    table = np.arange(12).reshape(3, 4)
    table[0, 1], table[1, 0], table[1, 1], table[2, 3] = 12, -1, 2 ** 31 - 1, -7        # (the last one holds no key)
    q = rand_i8(rng, (5, hq * d))
    attend(c, g, ref, q, hq, tq, lens, table, weights=True)
    torch.cuda.synchronize()
    assert c.poll_status() == -3 and c.poll_status() == 0
    table = np.arange(12).reshape(3, 4)
    cache = g.binding.Kv4Cache(cuda(ref.to_bytes()), d, page)

    def call(qs, lens, max_q, max_len):
        out = torch.full((5, hq * d), 55, dtype=torch.int8, device="cuda")
        c.kv4_attention(cache, cuda(q), cuda(np.array(qs, np.int32)), cuda(np.array(lens, np.int32)), cuda(table.astype(np.int32)),
                        g.binding.DevScale.of(*dyadic(1e-4)), ExpParams(17, 15), g.binding.DevScale.of(*dyadic(1 / 128)), max_q, max_len, out=out)
        torch.cuda.synchronize()
        return g.host(out)

    good = call([0, 1, 4, 5], [100, 64, 70], 3, 128)
    assert c.poll_status() == 0
    for qs, lens, max_q, max_len, same in (([0, 1, 4, 5], [100, 64, 2 ** 31 - 1], 3, 128, slice(0, 4)), ([0, 1, 4, 5], [-3, 64, 70], 3, 128, slice(1, 5)),
                                           ([0, 1, 4, 5], [100, 64, 70], 2, 128, slice(0, 1)), ([0, 1, 4, 2 ** 30], [100, 64, 70], 3, 128, slice(0, 4)),
                                           ([-5, 1, 4, 5], [100, 64, 70], 3, 128, slice(1, 5)), ([0, 1, 4, -2 ** 31], [100, 64, 70], 3, 128, slice(0, 4))):
        got = call(qs, lens, max_q, max_len)
        assert c.poll_status() == -3, (qs, lens)
        assert np.array_equal(got[same], good[same]), (qs, lens)


# ---- eviction ----

@pytest.mark.parametrize("d,page,hk", [(64, 32, 1), (128, 64, 3), (64, 256, 5), (128, 128, 2)])
@pytest.mark.parametrize("keep,sinks,recent", [(1, 0, 0), (1, 1, 0), (40, 4, 16), (100, 0, 100), (33, 33, 0), (255, 1, 3), (600, 4, 64)])
def test_evict_parity(d, page, hk, keep, sinks, recent):
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(d + page + keep)
    lens = [0, 1, keep - 1, keep, keep + 1, 300, 1029, 2500]
    B, ps, pd = len(lens), -(-2500 // page), -(-keep // page)
    w = rng.integers(0, 50, (B, hk, 2500)) << rng.integers(0, 45, (B, hk, 2500))
    w[5], w[6, :, ::2] = 7, 2 ** 62                                 # all equal; half of them equal at the top
    for in_place in (False, True):
        ref = filled(rng, B * (ps + pd), hk, d, page)
        order = rng.permutation(B * (ps + pd))
        table, dst = order[:B * ps].reshape(B, ps).astype(np.int32), order[B * ps:].reshape(B, pd).astype(np.int32)
        cache = g.binding.Kv4Cache(cuda(ref.to_bytes()), d, page)
        dw, dl, dt = cuda(w), cuda(np.array(lens, np.int32)), cuda(table)
        if in_place:
            kept, new = c.kv4_evict(cache, dw, dl, dt, keep, sinks, recent, 2500, new_lens=dl)
            wo = dw
        else:
            wo = torch.full((B, hk, pd * page + 3), -5, dtype=torch.int64, device="cuda")
            kept, new = c.kv4_evict(cache, dw, dl, dt, keep, sinks, recent, 2500, dst_table=cuda(dst), weights_out=wo)
        wk, wn, ww, pool = D.evict(ref, w, lens, table, table if in_place else dst, wo.shape[2], keep, sinks, recent)
        g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
        g.assert_equal(g.host(new), wn.astype(np.int32), "new lens")
        g.assert_equal(g.host(wo), ww, "weights")
        g.assert_equal(g.host(cache.pool), pool, "pool")
        assert c.poll_status() == 0


def test_evict_any_weights():
    """Negative weights and the ends of int64 order like any others."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(8)
    L, keep = 1500, 700
    w = rng.choice([-2 ** 63, 2 ** 63 - 1, -1, 0, 1, 255, 256, -256, 2 ** 40], (2, 2, L))
    ref = filled(rng, 2 * 12, 2, 64, 128)
    table = np.arange(24).reshape(2, 12).astype(np.int32)
    cache, dw = g.binding.Kv4Cache(cuda(ref.to_bytes()), 64, 128), cuda(w)
    kept, _ = c.kv4_evict(cache, dw, cuda(np.array([L, L - 1], np.int32)), cuda(table), keep, 2, 9, L)
    wk, _, ww, pool = D.evict(ref, w, [L, L - 1], table, table, L, keep, 2, 9)
    g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
    g.assert_equal(g.host(dw), ww, "weights")
    g.assert_equal(g.host(cache.pool), pool, "pool")


def test_evict_long():
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(9)
    L, keep, page = 70001, 30011, 256
    np_ = -(-L // page)
    w = (rng.standard_exponential((1, 2, L)) ** 4 * 1e6).astype(np.int64)
    for in_place in (True, False):
        ref = filled(rng, 2 * np_, 2, 64, page)
        table, dst = np.arange(np_, dtype=np.int32)[None], np.arange(np_, 2 * np_, dtype=np.int32)[None]
        cache, dw = g.binding.Kv4Cache(cuda(ref.to_bytes()), 64, page), cuda(w)
        wo = dw if in_place else torch.empty_like(dw)
        to = table if in_place else dst
        kept, _ = c.kv4_evict(cache, dw, cuda(np.array([L], np.int32)), cuda(table), keep, 4, 500, L, dst_table=None if in_place else cuda(dst), weights_out=wo)
        wk, _, ww, pool = D.evict(ref, w, [L], table, to, L, keep, 4, 500)
        g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
        g.assert_equal(g.host(wo), ww, "weights")
        g.assert_equal(g.host(cache.pool), pool, "pool")


def test_evict_reports_lengths_and_pages():
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(10)
    ref = filled(rng, 8, 2, 64, 32)
    w = rng.integers(0, 1000, (2, 2, 128))
    table = np.arange(8).reshape(2, 4).astype(np.int32)
    bad = table.copy()
    bad[1, 2] = 8
    for lens, t in (([200, 100], table), ([100, -4], table), ([100, 128], bad)):
        cache = g.binding.Kv4Cache(cuda(ref.to_bytes()), 64, 32)
        kept, new = c.kv4_evict(cache, cuda(w), cuda(np.array(lens, np.int32)), cuda(t), 50, 1, 1, 128)
        torch.cuda.synchronize()
        assert c.poll_status() == -3
        assert g.host(new).tolist() == [min(50, max(0, min(n, 128))) for n in lens]


# ---- as they are used ----

def test_a_decoder_step_and_a_graph_of_it():
    """Prompt, then tokens one by one: norm, QKV Dense, append, attention, output Dense, norm; then eviction and one more token.
    Each operator's reference takes the same bytes as its kernel; the token step is then captured and replayed with the same result."""
    g = _g()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = g.binding.Context(0, stream)
        rng = np.random.default_rng(21)
        d, hq, hk, page, pages, steps, prompt = 64, 6, 2, 32, 8, 6, 70
        Dm = hq * d
        wqkv, wo = rand_i8(rng, ((hq + 2 * hk) * d, Dm), 33), rand_i8(rng, (Dm, Dm), 33)
        acc = np.sqrt(Dm) * 32 * 33
        s_qkv, s_o = scale_channels(rng.uniform(25, 35, len(wqkv)) / acc), scale_channels(rng.uniform(8, 12, Dm) / acc)
        gamma = scale_channels(rng.uniform(28, 36, Dm) * np.sqrt(Dm) / 2 ** 20)
        unit, rs = Scale(*dyadic(0.5)), Scale(*dyadic(0.9))
        qk, pv = dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40)), dyadic(1 / 128)
        B = g.binding
        D_ = {n: B.DevScale(s, "cuda") for n, s in dict(qkv=s_qkv, o=s_o, gamma=gamma, unit=unit, rs=rs).items()}
        dqk, dpv, dwqkv, dwo = B.DevScale.of(*qk), B.DevScale.of(*pv), cuda(wqkv), cuda(wo)
        cache = B.Kv4Cache.empty(pages, hk, d, page, "cuda")
        cache.pool.copy_(cuda(D.Cache(pages, hk, d, page).to_bytes()))
        ref = D.Cache(pages, hk, d, page)
        table = np.array([[3, 0, 7, 2, 5]])
        dtable = cuda(table.astype(np.int32))
        weights = torch.zeros((1, hk, 160), dtype=torch.int64, device="cuda")
        w_ref = np.zeros((1, hk, 160), np.int64)

        def gpu(x, stream_in, slots, qs, lens):
            a = c.rmsnorm(x, D_["gamma"], x_scale=D_["unit"], res=stream_in, res_scale=D_["rs"], sum_out=stream_in)
            qkv = c.linear(a, dwqkv, None, D_["qkv"])
            c.kv4_append(cache, qkv[:, Dm:Dm + hk * d], qkv[:, Dm + hk * d:], slots)
            o = c.kv4_attention(cache, qkv[:, :Dm], qs, lens, dtable, dqk, ExpParams(17, 15), dpv, x.shape[0], 160, weights=weights)
            return c.linear(o, dwo, None, D_["o"], res=stream_in, res_scale=D_["rs"])

        def cpu(x, stream_in, slots, n, length):
            a, _, h = D.rmsnorm(x, (gamma.mult, gamma.shift), 20, (unit.mult, unit.shift), stream_in, (rs.mult, rs.shift))
            qkv = O.linear(a.astype(np.int8), wqkv, None, s_qkv)
            ref.append(qkv[:, Dm:Dm + hk * d], qkv[:, Dm + hk * d:], slots)
            nonlocal w_ref
            o, w_ref = D.attention(ref, qkv[:, :Dm], hq, [0, n], [length], table, qk, 17, 15, pv, np.zeros((n, Dm)), w_ref)
            return O.linear(o.astype(np.int8), wo, None, s_o, res=h.astype(np.int8), res_scale=rs), h

        def slots_of(j):
            return table[0][j // page] * page + j % page

        length = 0
        for step in range(steps):
            n = prompt if step == 0 else 1
            x, h = rand_i8(rng, (n, Dm)), rand_i8(rng, (n, Dm), 20)
            slots = slots_of(np.arange(length, length + n)).astype(np.int64)
            length += n
            dh = cuda(h)
            got = gpu(cuda(x), dh, cuda(slots), cuda(np.array([0, n], np.int32)), cuda(np.array([length], np.int32)))
            want, hh = cpu(x, h, slots, n, length)
            stream.synchronize()
            g.assert_equal(g.host(dh), hh.astype(np.int8), f"stream, step {step}")
            g.assert_equal(g.host(cache.pool), ref.to_bytes(), f"pool, step {step}")
            g.assert_equal(g.host(got), want, f"step {step}")
            g.assert_equal(g.host(weights), w_ref, f"weights, step {step}")
        kept, new = c.kv4_evict(cache, weights, cuda(np.array([length], np.int32)), dtable, 40, 4, 16, 160)
        wk, wn, w_ref, _ = D.evict(ref, w_ref, [length], table, table, 160, 40, 4, 16)
        g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
        g.assert_equal(g.host(cache.pool), ref.to_bytes(), "pool behind eviction")
        length = int(g.host(new)[0])
        # one more token, twice: launched, and as a graph that is replayed on new inputs
        bx, bh, bs = cuda(rand_i8(rng, (1, Dm))), cuda(rand_i8(rng, (1, Dm), 20)), cuda(slots_of(np.array([length])).astype(np.int64))
        bq, bl = cuda(np.array([0, 1], np.int32)), cuda(np.array([length + 1], np.int32))
        graph = torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            out = gpu(bx, bh, bs, bq, bl)
        for i in range(3):
            x, h = rand_i8(rng, (1, Dm)), rand_i8(rng, (1, Dm), 20)
            slots = slots_of(np.array([length])).astype(np.int64)
            length += 1
            for t, a in ((bx, x), (bh, h), (bs, slots), (bl, np.array([length], np.int32))):
                t.copy_(cuda(a))
            graph.replay()
            stream.synchronize()
            want, _ = cpu(x, h, slots, 1, length)
            g.assert_equal(g.host(out), want, f"replay {i}")
            g.assert_equal(g.host(weights), w_ref, f"weights, replay {i}")
        assert c.poll_status() == 0
        c.close()


# ---- what the calls allow and the tests above do not make ----

def test_two_contexts_at_once():
    """Clusters of two streams on the GPU at the same time, each with a context of its own."""
    g = _g()
    rng = np.random.default_rng(31)
    d, page, hk, hq, L = 128, 64, 4, 8, 20000
    np_ = -(-L // page)
    ref = filled(rng, np_, hk, d, page)
    table = rng.permutation(np_)[None]
    pool = cuda(ref.to_bytes())
    qk, pv = dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40)), dyadic(1 / 128)
    runs = []
    for i in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            q, length = rand_i8(rng, (1, hq * d)), L - 777 * i
            runs.append(dict(s=s, c=g.binding.Context(0, s), q=q, length=length, dq=cuda(q), qs=cuda(np.array([0, 1], np.int32)),
                             lens=cuda(np.array([length], np.int32)), table=cuda(table.astype(np.int32)),
                             out=torch.zeros((1, hq * d), dtype=torch.int8, device="cuda"), w=torch.zeros((1, hk, L), dtype=torch.int64, device="cuda")))
        s.synchronize()
    for _ in range(10):
        for r in runs:
            with torch.cuda.stream(r["s"]):
                r["c"].kv4_attention(g.binding.Kv4Cache(pool, d, page), r["dq"], r["qs"], r["lens"], r["table"], g.binding.DevScale.of(*qk),
                                     ExpParams(17, 15), g.binding.DevScale.of(*pv), 1, L, out=r["out"], weights=r["w"])
    torch.cuda.synchronize()
    for r in runs:
        want, w = D.attention(ref, r["q"], hq, [0, 1], [r["length"]], table, qk, 17, 15, pv, np.zeros((1, hq * d)), np.zeros((1, hk, L), np.int64))
        g.assert_equal(g.host(r["out"]), want.astype(np.int8), "out")
        g.assert_equal(g.host(r["w"]), 10 * w, "weights")
        assert r["c"].poll_status() == 0
        r["c"].close()


def test_graph_of_a_split_sequence_and_its_eviction():
    """Attention by clusters, then eviction in place, captured once and replayed while the length on the device changes."""
    g = _g()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = g.binding.Context(0, stream)
        rng = np.random.default_rng(32)
        d, page, hk, hq, L, keep = 64, 64, 2, 8, 17000, 9000
        np_ = -(-L // page)
        ref = filled(rng, np_, hk, d, page)
        table = rng.permutation(np_)[None].astype(np.int32)
        cache = g.binding.Kv4Cache(cuda(ref.to_bytes()), d, page)
        qk, pv = dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40)), dyadic(1 / 128)
        dqk, dpv, dtable = g.binding.DevScale.of(*qk), g.binding.DevScale.of(*pv), cuda(table)
        q = rand_i8(rng, (1, hq * d))
        dq, qs, lens = cuda(q), cuda(np.array([0, 1], np.int32)), cuda(np.array([L], np.int32))
        out, w = torch.zeros((1, hq * d), dtype=torch.int8, device="cuda"), torch.zeros((1, hk, L), dtype=torch.int64, device="cuda")
        kept, new = torch.zeros((1, hk, keep), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.kv4_attention(cache, dq, qs, lens, dtable, dqk, ExpParams(17, 15), dpv, 1, L, out=out, weights=w)
            c.kv4_evict(cache, w, lens, dtable, keep, 4, 100, L, kept=kept, new_lens=new)
        ww = np.zeros((1, hk, L), np.int64)
        for length in (L, 9000, 8999, 9500, 40, 0):
            lens.copy_(cuda(np.array([length], np.int32)))
            graph.replay()
            stream.synchronize()
            want, ww = D.attention(ref, q, hq, [0, 1], [length], table, qk, 17, 15, pv, np.zeros((1, hq * d)), ww)
            wk, wn, ww, pool = D.evict(ref, ww, [length], table, table, L, keep, 4, 100)
            g.assert_equal(g.host(out), want.astype(np.int8), f"out, {length}")
            g.assert_equal(g.host(kept), wk.astype(np.int32), f"kept, {length}")
            g.assert_equal(g.host(w), ww, f"weights, {length}")
            g.assert_equal(g.host(cache.pool), pool, f"pool, {length}")
            assert int(new) == wn[0]
        assert c.poll_status() == 0
        c.close()


@pytest.mark.parametrize("pages_in_place,weights_in_place", [(True, False), (False, True)])
def test_evict_with_only_one_of_two_in_place(pages_in_place, weights_in_place):
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(33)
    L, keep, page, hk, B = 1100, 300, 32, 3, 2
    ps, pd = -(-L // page), -(-keep // page)
    ref = filled(rng, B * (ps + pd), hk, 128, page)
    order = rng.permutation(B * (ps + pd)).astype(np.int32)
    table, dst = order[:B * ps].reshape(B, ps), order[B * ps:].reshape(B, pd)
    w = rng.integers(0, 10 ** 6, (B, hk, L))
    cache, dw, dt = g.binding.Kv4Cache(cuda(ref.to_bytes()), 128, page), cuda(w), cuda(table)
    wo = dw if weights_in_place else torch.full((B, hk, keep + 1), -1, dtype=torch.int64, device="cuda")
    kept, _ = c.kv4_evict(cache, dw, cuda(np.array([L, 299], np.int32)), dt, keep, 3, 7, L, dst_table=dt if pages_in_place else cuda(dst), weights_out=wo)
    wk, _, ww, pool = D.evict(ref, w, [L, 299], table, table if pages_in_place else dst, wo.shape[2], keep, 3, 7)
    g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
    g.assert_equal(g.host(wo), ww, "weights")
    g.assert_equal(g.host(cache.pool), pool, "pool")


def test_the_binding_refuses_what_the_library_would_misread():
    """Types, shapes, strides and devices: refused before anything is launched."""
    g, c = _g(), _g().ctx()
    B = g.binding
    z = lambda *s, t=torch.int8: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    one = B.DevScale.of(2 ** 30, 40)
    host_scale = B.DevScale(Scale(np.full(64, 2 ** 30, np.int32), np.full(64, 40, np.uint8)), "cpu")
    x, cache = z(4, 64), B.Kv4Cache.empty(4, 2, 64, 32, "cuda")
    lens, qs, table, w = z(2, t=torch.int32), z(3, t=torch.int32), z(2, 2, t=torch.int32), z(2, 2, 64, t=torch.int64)
    q, smax = z(2, 256), ExpParams(17, 15)
    att = lambda **k: c.kv4_attention(**{**dict(cache=cache, q=q, q_start=qs, lens=lens, table=table, qk_scale=one, smax=smax, pv_scale=one, max_q=1, max_len=64), **k})  # noqa: E731
    evi = lambda **k: c.kv4_evict(**{**dict(cache=cache, weights=w, lens=lens, table=table, keep=40, sinks=1, recent=1, max_len=64), **k})  # noqa: E731
    app = lambda **k: c.kv4_append(**{**dict(cache=cache, k=z(4, 128), v=z(4, 128), slots=z(4, t=torch.int64)), **k})  # noqa: E731
    nrm = lambda **k: c.rmsnorm(**{**dict(x=x, gamma_scale=one), **k})  # noqa: E731
    before = c.launch_count()
    for f, bad in ((nrm, [dict(x=x.cpu()), dict(x=x.half()), dict(x=z(64)), dict(x=z(64, 64).t()[:4]), dict(out=z(4, 48)), dict(out=z(4, 64, t=torch.int32)),
                          dict(res=x), dict(res=z(3, 64), x_scale=one, res_scale=one), dict(sum_out=x), dict(row_max=z(3, t=torch.int32)),
                          dict(row_max=z(4, t=torch.int64)), dict(gamma_scale=host_scale), dict(res=x, x_scale=host_scale, res_scale=one),
                          dict(res=x, x_scale=one, res_scale=one, sum_out=z(4, 64, t=torch.int32))]),
                   (app, [dict(k=z(4, 64), v=z(4, 64)), dict(v=z(3, 128)), dict(slots=z(3, t=torch.int64)), dict(slots=z(4, t=torch.int32)),
                          dict(slots=z(4, t=torch.int64).cpu()), dict(k=z(4, 256)[:, ::2]), dict(slots=z(8, t=torch.int64)[::2])]),
                   (att, [dict(q=q.cpu()), dict(q=z(2, 100)), dict(out=z(3, 256)), dict(q_start=z(2, t=torch.int32)), dict(q_start=z(3, t=torch.int64)),
                          dict(lens=lens.cpu()), dict(table=z(3, 2, t=torch.int32)), dict(table=z(2, 1, t=torch.int32)), dict(max_len=65),
                          dict(table=z(2, 2, t=torch.int64)), dict(weights=z(2, 1, 64, t=torch.int64)), dict(weights=z(2, 2, 64, t=torch.int32)),
                          dict(weights=z(2, 2, 128, t=torch.int64)[:, :, :64])]),
                   (evi, [dict(weights=z(1, 2, 64, t=torch.int64)), dict(weights=w[:, :, ::2]), dict(table=table.t()), dict(max_len=65),
                          dict(dst_table=z(2, 1, t=torch.int32)), dict(weights_out=z(2, 3, 64, t=torch.int64)), dict(kept=z(2, 2, 39, t=torch.int32)),
                          dict(new_lens=z(3, t=torch.int32)), dict(lens=lens.cpu())])):
        for k in bad:
            with pytest.raises(ValueError):
                f(**k)
    for make in (lambda: B.Kv4Cache(z(4, 2, 32 * 67), 64, 32), lambda: B.Kv4Cache(z(4, 2, 32 * 67 + 1, t=torch.uint8), 64, 32),
                 lambda: B.Kv4Cache(z(4, 2, 48 * 67, t=torch.uint8), 64, 48)):
        with pytest.raises(ValueError):
            make()
    with pytest.raises(B.IvitError):
        evi(weights_out=z(2, 2, 39, t=torch.int64))
    assert c.launch_count() == before
    torch.cuda.synchronize()
    assert c.poll_status() == 0


def _calls_that_make_their_outputs(c, g):
    """name -> (a call that is given no output, its first output's bytes), on inputs that stay as they are."""
    rng = np.random.default_rng(41)
    B, one = g.binding, g.binding.DevScale.of(*dyadic(0.01))
    rows, d, page, hk, L = 1500, 64, 32, 2, 300
    x, w = cuda(rand_i8(rng, (rows, 1024))), cuda(rand_i8(rng, (1024, 1024)))
    ref = filled(rng, 20, hk, d, page)
    cache = B.Kv4Cache(cuda(ref.to_bytes()), d, page)
    q, qs, lens = cuda(rand_i8(rng, (rows, 4 * d))), cuda(np.array([0, 100], np.int32)), cuda(np.array([L], np.int32))
    table, dst = cuda(np.arange(10, dtype=np.int32)[None]), cuda(np.arange(10, 20, dtype=np.int32)[None])
    weights, wo = cuda(rng.integers(0, 10 ** 6, (1, hk, L))), torch.zeros((1, hk, 320), dtype=torch.int64, device="cuda")
    qk, pv, gelu = B.DevScale.of(*dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40))), B.DevScale.of(*dyadic(1 / 128)), ExpParams(17, 15)
    nb = cuda(rand_i8(rng, (9, 90, 64)))
    index = cuda(rng.integers(0, rows, 700).astype(np.int32))
    return {
        "rmsnorm": (lambda: c.rmsnorm(x, one), rows * 1024),
        "kv4_attention": (lambda: c.kv4_attention(cache, q, qs, lens, table, qk, gelu, pv, 100, L), rows * 4 * d),
        "kv4_evict": (lambda: c.kv4_evict(cache, weights, lens, table, 200, 4, 16, L, dst_table=dst, weights_out=wo)[0], 4 * hk * 200),
        "linear": (lambda: c.linear(x, w, None, one), rows * 1024),
        "matmul": (lambda: c.matmul(nb, nb, True, one), 9 * 90 * 96),
        "layernorm": (lambda: c.layernorm(x, one, None), rows * 1024),
        "gather_rows": (lambda: c.gather_rows(x, index), 700 * 1024),
        "token_mean": (lambda: c.token_mean(x, 3, one), 500 * 1024),
    }


@pytest.mark.parametrize("name", ["rmsnorm", "kv4_attention", "kv4_evict", "linear", "matmul", "layernorm", "gather_rows", "token_mean"])
def test_outputs_that_a_call_makes_belong_to_the_context_s_stream(name):
    """A context with a stream of its own, while another one is current and busy: what the call does to a new output may not wait there (zeros that
    land behind the kernel), and its memory may not be a block that the current stream has still to read."""
    g = _g()
    side = torch.cuda.Stream()
    c = g.binding.Context(0, side)
    call, nbytes = _calls_that_make_their_outputs(c, g)[name]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        want = [g.host(call()) for _ in range(2)][1]
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)                                   # (20 ms)
    got = call()
    torch.cuda.synchronize()
    g.assert_equal(g.host(got), want, "behind a busy stream")
    del got
    for _ in range(3):
        old = torch.full((nbytes,), 77, dtype=torch.int8, device="cuda")
        copy = torch.empty_like(old)
        torch.cuda.synchronize()
        torch.cuda._sleep(40_000_000)
        copy.copy_(old)
        del old
        got = call()
        torch.cuda.synchronize()
        assert (copy == 77).all()
        g.assert_equal(g.host(got), want, "beside a busy stream")
        del got
    # what the current stream still reads of an output that the caller has dropped is not the next call's output
    side.synchronize()
    for _ in range(3):
        got = call()
        torch.cuda.current_stream().wait_stream(side)
        copy = torch.empty_like(got)
        torch.cuda._sleep(40_000_000)
        copy.copy_(got)
        got = None
        with torch.cuda.stream(side):
            junk = [torch.full((nbytes,), 77, dtype=torch.int8, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        g.assert_equal(g.host(copy), want, "read by a busy stream")
        del junk
    assert c.poll_status() == 0
    c.close()


@pytest.mark.parametrize("B", [1, 2])
@pytest.mark.parametrize("cols,dst_cols", [(40, 5), (5, 40), (40, 40)])
def test_evict_in_place_by_columns_of_one_table(B, cols, dst_cols):
    """The table's first columns name where the rows go: in place, whatever the columns and however few the sequences."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(43)
    L, keep, page, hk = 150, 70, 32, 2
    ref = filled(rng, B * 5 + 1, hk, 64, page)
    table = np.full((B, 40), -1, np.int32)
    table[:, :5] = rng.permutation(B * 5).reshape(B, 5)
    w, lens = rng.integers(0, 10 ** 6, (B, hk, L)), [L, 90][:B]
    cache, dw, dt = g.binding.Kv4Cache(cuda(ref.to_bytes()), 64, page), cuda(w), cuda(table)
    kept, _ = c.kv4_evict(cache, dw, cuda(np.array(lens, np.int32)), dt[:, :cols], keep, 3, 7, L, dst_table=dt[:, :dst_cols])
    wk, _, ww, pool = D.evict(ref, w, lens, table, table, L, keep, 3, 7)
    g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
    g.assert_equal(g.host(dw), ww, "weights")
    g.assert_equal(g.host(cache.pool), pool, "pool")
    assert c.poll_status() == 0


def test_the_first_attention_of_a_context_is_captured():
    """A context that has made no call: its first attention, by a cluster, goes into a graph; a second context's runs at once."""
    g = _g()
    rng = np.random.default_rng(47)
    d, page, hk, hq, L = 64, 64, 2, 4, 5000
    np_ = -(-L // page)
    ref = filled(rng, np_, hk, d, page)
    table, q = rng.permutation(np_)[None], rand_i8(rng, (1, hq * d))
    qk, pv = dyadic(25.0 / (8 * np.sqrt(d) * 32 * 40)), dyadic(1 / 128)
    want, _ = D.attention(ref, q, hq, [0, 1], [L], table, qk, 17, 15, pv, np.zeros((1, hq * d)))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        cache = g.binding.Kv4Cache(cuda(ref.to_bytes()), d, page)
        args = (cache, cuda(q), cuda(np.array([0, 1], np.int32)), cuda(np.array([L], np.int32)), cuda(table.astype(np.int32)), g.binding.DevScale.of(*qk),
                ExpParams(17, 15), g.binding.DevScale.of(*pv), 1, L)
        out = torch.full((1, hq * d), 55, dtype=torch.int8, device="cuda")
        c = g.binding.Context(0, stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.kv4_attention(*args, out=out)
        stream.synchronize()
        assert (out == 55).all()
        graph.replay()
        stream.synchronize()
        g.assert_equal(g.host(out), want.astype(np.int8), "replayed")
        other = g.binding.Context(0, stream)
        out.fill_(55)
        other.kv4_attention(*args, out=out)
        stream.synchronize()
        g.assert_equal(g.host(out), want.astype(np.int8), "launched")
        for x in (c, other):
            assert x.poll_status() == 0
            x.close()


# rows that are taken several at a time (GROUPED: 8, with an int32 tensor or row scales 4), at widths whose threads' words are all there (C / 4 a
# multiple of 64) and at others, the last group not full
GROUPED = [(3601, 132), (1999, 1000), (1999, 2048), (901, 4092)]


@pytest.mark.parametrize("x32,h32", [(0, None), (1, None), (0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("rows,C", GROUPED)
def test_rmsnorm_groups_of_rows(rows, C, x32, h32):
    g, c = _g(), _g().ctx()
    sms, R = torch.cuda.get_device_properties(0).multi_processor_count, 8
    assert rows >= 3 * sms and (rows * (C // 4) >= 275 * R * sms or rows >= 3 * R * sms) and rows % 4   # (the rule, at its largest R)
    rng = np.random.default_rng(rows + C + 7 * x32 + 3 * (h32 or 0))
    for kind in ("ordinary", "extreme"):
        x, res = norm_case(rng, rows, C, x32, h32 or 0, kind)
        x[-1], res[-2] = x[-1][::-1], 0
        xs = scale_channels(rng.uniform(0.5, 1.5, C) * ((500.0 if h32 else 10.0) / (20000.0 if x32 else 1100.0)))
        rs = Scale(*dyadic(0.96875))
        for dynamic, M_ln, ratio in ((False, 20, 32.0 * np.sqrt(C) / 2 ** 20), (True, 22, 0.4)):
            gs = scale_channels(rng.uniform(0.8, 1.1, C) * min(ratio, 0.9))
            want, top, total = D.rmsnorm(x, (gs.mult, gs.shift), M_ln, (xs.mult, xs.shift), None if h32 is None else res, (rs.mult, rs.shift), h32 == 1,
                                         dynamic)
            sums = None if h32 is None else g.dev(np.zeros_like(res))
            rm = torch.full((rows,), -1, dtype=torch.int32, device="cuda") if dynamic else None
            got = c.rmsnorm(g.dev(x), g.binding.DevScale(gs, "cuda"), x_scale=g.binding.DevScale(xs, "cuda"), res=None if h32 is None else g.dev(res),
                            res_scale=None if h32 is None else g.binding.DevScale(rs, "cuda"), M_ln=M_ln, sum_out=sums, row_max=rm)
            what = f"{kind}, dynamic {dynamic}"
            g.assert_equal(g.host(got), want.astype(np.int8), what)
            if dynamic:
                g.assert_equal(g.host(rm), top.astype(np.int32), what + " row_max")
            if h32 is not None:
                g.assert_equal(g.host(sums), total.astype(res.dtype), what + " sum")
    assert c.poll_status() == 0


@pytest.mark.parametrize("h32", [0, 1])
@pytest.mark.parametrize("rows,C", GROUPED)
def test_rmsnorm_groups_leave_the_rest_alone(rows, C, h32):
    """The stream in place: columns past C and rows past the last keep what they held, the others get their sums once."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(rows + h32)
    x, res = norm_case(rng, rows, C, 0, h32, "ordinary")
    ld = (C + 15) // 16 * 16 + 16
    dt = torch.int32 if h32 else torch.int8
    scale = Scale(*dyadic(0.01))
    s = g.binding.DevScale(scale, "cuda")
    for dynamic in (False, True):
        bx = torch.full((rows + 9, ld), 77, dtype=torch.int8, device="cuda")
        br, bo, rm = bx.clone().to(dt), bx.clone(), torch.full((rows + 9,), 77, dtype=torch.int32, device="cuda")
        bx[:rows, :C], br[:rows, :C] = cuda(x), cuda(res)
        c.rmsnorm(bx[:rows, :C], s, x_scale=s, res=br[:rows, :C], res_scale=s, sum_out=br[:rows, :C], out=bo[:rows, :C], row_max=rm[:rows] if dynamic else None)
        want, top, total = D.rmsnorm(x, (scale.mult, scale.shift), 20, (scale.mult, scale.shift), res, (scale.mult, scale.shift), h32 == 1, dynamic)
        g.assert_equal(g.host(bo[:rows, :C]), want.astype(np.int8), "out")
        g.assert_equal(g.host(br[:rows, :C]), total.astype(res.dtype), "stream")
        g.assert_equal(g.host(bx[:rows, :C]), x, "x")
        for t in (bx, br, bo):
            assert (t[rows:] == 77).all() and (t[:, C:] == 77).all()
        assert (rm[rows if dynamic else 0:] == 77).all()
        if dynamic:
            g.assert_equal(g.host(rm[:rows]), top.astype(np.int32), "row_max")


def weights_of(kind, rng, L):
    """Weights whose threshold falls where the kernel's first digit (bit length and five bits) does not tell it."""
    if kind == "equal":                # one value, far above the small ones
        return np.full(L, 3 << 40)
    if kind == "equal_and_others":     # as many as are wanted and more of one value, a few above and below in other digits
        w = np.full(L, (1 << 50) + 12345)
        w[rng.permutation(L)[:L // 20]] = rng.integers(0, 1 << 62, L // 20)
        return w
    if kind == "one_digit":            # all of one digit, most of them different, some equal ones
        return (1 << 40) + rng.integers(0, 1 << 34, L) // 3 * 3
    if kind == "one_digit_ties":       # few values, of one digit: ties at the threshold
        return (1 << 40) + rng.integers(0, 3, L) * 65537
    if kind == "low_bytes":            # equal but for the last byte
        return (1 << 55) + rng.integers(0, 200, L)
    if kind == "negative":             # nearly all below zero: the threshold too
        w = -rng.integers(1, 1 << 62, L)
        w[rng.permutation(L)[:40]] = rng.integers(0, 1 << 40, 40)
        return w
    if kind == "negative_equal":       # all of them the least value
        return np.full(L, -2 ** 63)
    if kind == "negative_and_zero":    # zeros and negative ones share the first digit
        return np.where(rng.random(L) < 0.1, 0, -rng.integers(1, 5, L))
    # few_negative: at most 1024 below one, the threshold among them
    w = rng.integers(1 << 20, 1 << 60, L)
    w[rng.permutation(L)[:700]] = -rng.integers(0, 9, 700)
    return w


KINDS = ["equal", "equal_and_others", "one_digit", "one_digit_ties", "low_bytes", "negative", "negative_equal", "negative_and_zero", "few_negative"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("L", [2900, 16384, 16385, 20003])      # (keys in registers up to 16384, else read again)
def test_evict_selects_within_one_digit(L, kind):
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(L + len(kind))
    page, hk, sinks, recent = 256, 2, 3, 50
    keep = L - 300 if kind == "few_negative" else L // 2
    np_ = -(-L // page)
    w = np.stack([weights_of(kind, rng, L) for _ in range(2 * hk)]).reshape(2, hk, L).astype(np.int64)
    w[:, :, :sinks], w[:, :, L - 500:] = 2 ** 63 - 1, np.where(rng.random(500) < 0.5, -2 ** 63, w[:, :, L - 500:])   # (not candidates; another length's are)
    lens = [L, L - 400]
    for in_place in (True, False):
        ref = filled(rng, 4 * np_, hk, 64, page)
        table, dst = np.arange(2 * np_, dtype=np.int32).reshape(2, np_), np.arange(2 * np_, 4 * np_, dtype=np.int32).reshape(2, np_)
        cache, dw = g.binding.Kv4Cache(cuda(ref.to_bytes()), 64, page), cuda(w)
        wo = dw if in_place else torch.empty_like(dw)
        kept, new = c.kv4_evict(cache, dw, cuda(np.array(lens, np.int32)), cuda(table), keep, sinks, recent, L,
                                dst_table=None if in_place else cuda(dst), weights_out=wo)
        wk, wn, ww, pool = D.evict(ref, w, lens, table, table if in_place else dst, L, keep, sinks, recent)
        g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
        g.assert_equal(g.host(new), wn.astype(np.int32), "new lens")
        g.assert_equal(g.host(wo), ww, "weights")
        g.assert_equal(g.host(cache.pool), pool, "pool")
    assert c.poll_status() == 0


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_evict_moves_nothing_from_or_to_pages_that_are_not_there(d, in_place):
    """Rows of source or destination pages outside the pool: no byte of them is written, all others move; kept, weights and lengths as ever."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(d)
    page, hk, keep, sinks, recent, L = 32, 2, 100, 2, 9, 200
    lens = [200, 200, 77, 260, -4]                      # (the last two: past max_len, and none)
    B, ps, pd = len(lens), 7, 4
    before = rng.integers(0, 256, (B * (ps + pd), hk, page * (d + d // 32 + 1))).astype(np.uint8)
    order = rng.permutation(B * (ps + pd)).astype(np.int32)
    table, dst = order[:B * ps].reshape(B, ps).copy(), order[B * ps:].reshape(B, pd).copy()
    table[0, 1], table[0, 4], table[1, 0], table[2, 2], table[2, 6] = len(before), -1, 2 ** 31 - 1, -2 ** 31, 12345   # (the last one holds no key)
    dst[1, 2], dst[2, 0], dst[3, 3] = -1, len(before), 2 ** 31 - 1
    w = rng.integers(0, 10 ** 6, (B, hk, L))
    cache, dw, dt = g.binding.Kv4Cache(cuda(before), d, page), cuda(w), cuda(table)
    wo = dw if in_place else torch.full((B, hk, pd * page), -5, dtype=torch.int64, device="cuda")
    kept, new = c.kv4_evict(cache, dw, cuda(np.array(lens, np.int32)), dt, keep, sinks, recent, L, dst_table=dt if in_place else cuda(dst), weights_out=wo)
    torch.cuda.synchronize()
    assert c.poll_status() == -3 and c.poll_status() == 0
    to = table if in_place else dst
    at = dict(kc=(0, d // 2), ks=(page * d // 2, d // 32), vc=(page * (d // 2 + d // 32), d // 2), vs=(page * (d + d // 32), 1))
    pool, wk, ww = before.copy(), np.full((B, hk, keep), -1), np.zeros((B, hk, wo.shape[2]), np.int64)
    for b in range(B):
        n = min(max(lens[b], 0), L)
        for h in range(hk):
            stay = list(range(n))
            if n > keep:
                best = sorted(range(sinks, n - recent), key=lambda j: (-w[b, h, j], j))[:keep - sinks - recent]
                stay = sorted(list(range(sinks)) + best + list(range(n - recent, n)))
            wk[b, h, :len(stay)], ww[b, h, :len(stay)] = stay, w[b, h, stay]
            for i, j in enumerate(stay):
                s, t = table[b, j // page], to[b, i // page]
                if 0 <= s < len(before) and 0 <= t < len(before):
                    for first, step in at.values():
                        pool[t, h, first + i % page * step:first + (i % page + 1) * step] = before[s, h, first + j % page * step:first + (j % page + 1) * step]
    g.assert_equal(g.host(kept), wk.astype(np.int32), "kept")
    g.assert_equal(g.host(new), np.array([min(keep, max(0, min(n, L))) for n in lens], np.int32), "new lens")
    g.assert_equal(g.host(wo), ww, "weights")
    g.assert_equal(g.host(cache.pool), pool, "pool")


@pytest.mark.parametrize("B,hk,G,L", [(40, 4, 2, 2700), (38, 8, 4, 4000), (128, 2, 3, 2600)])
def test_attention_longest_first(B, hk, G, L):
    """Heads of 128 in CTAs of sixteen warps that take the sequences longest first (40 blocks of 32 keys or more for each wave of CTAs): equal lengths, empty ones,
    bad ones, the longest at the end."""
    g, c = _g(), _g().ctx()
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert B <= 128 and B * hk > sms and -(-L // 32) >= 40 * -(-B * hk // sms)
    rng = np.random.default_rng(B)
    d, page = 128, 64
    lens = rng.integers(0, L + 1, B)
    lens[::4], lens[1], lens[-1] = L // 3, 0, L
    np_ = -(-L // page)
    ref = filled(rng, 60, hk, d, page)
    q, table = rand_i8(rng, (B, G * hk * d)), rng.integers(0, 60, (B, np_))
    for w in (False, True):
        attend(c, g, ref, q, G * hk, [1] * B, lens, table, weights=w, max_len=L)
    assert c.poll_status() == 0


def test_calls_without_rows_or_sequences():
    """Nothing to do: every operator takes it, launches nothing, and hands back tensors of the right shapes."""
    g, c = _g(), _g().ctx()
    B = g.binding
    z = lambda *s, t=torch.int8: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    one, cache, i32, i64 = B.DevScale.of(2 ** 30, 40), B.Kv4Cache.empty(4, 2, 64, 32, "cuda"), torch.int32, torch.int64
    before = c.launch_count()
    assert c.rmsnorm(z(0, 64), one).shape == (0, 64)
    assert c.rmsnorm(z(0, 64), one, x_scale=one, res=z(0, 64), res_scale=one, sum_out=z(0, 64), row_max=z(0, t=i32)).shape == (0, 64)
    c.kv4_append(cache, z(0, 128), z(0, 128), z(0, t=i64))
    att = lambda n, b: c.kv4_attention(cache, z(n, 256), z(b + 1, t=i32), z(b, t=i32), z(b, 2, t=i32), one, ExpParams(17, 15), one, 1, 64, weights=z(b, 2, 64, t=i64))  # noqa: E731
    assert att(0, 0).shape == (0, 256) and att(0, 3).shape == (0, 256) and att(3, 0).shape == (3, 256)
    for k in (dict(), dict(dst_table=z(0, 5, t=i32)), dict(dst_table=z(0, 5, t=i32), weights_out=z(0, 2, 40, t=i64))):
        kept, new = c.kv4_evict(cache, z(0, 2, 64, t=i64), z(0, t=i32), z(0, 2, t=i32), 40, 1, 1, 64, **k)
        assert kept.shape == (0, 2, 40) and new.shape == (0,)
    assert c.launch_count() == before
    torch.cuda.synchronize()
    assert c.poll_status() == 0


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_without_keys(in_place):
    """Sequences that have no keys yet, in a call that is sized for none: tables and weights without columns."""
    g, c = _g(), _g().ctx()
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    pool = torch.full((4, 2, 32 * 67), 99, dtype=torch.uint8, device="cuda")
    cache, keep = g.binding.Kv4Cache(pool, 64, 32), 40
    table = z(3, 0)
    wo = torch.full((3, 2, 45), -5, dtype=torch.int64, device="cuda")
    kept, new = c.kv4_evict(cache, z(3, 2, 0, t=torch.int64), z(3), table, keep, 4, 16, 0, dst_table=None if in_place else z(3, 2), weights_out=wo)
    assert (kept == -1).all() and (new == 0).all() and (wo == 0).all() and (pool == 99).all()
    torch.cuda.synchronize()
    assert c.poll_status() == 0


@pytest.mark.parametrize("wide", [0, 1])
@pytest.mark.parametrize("rows,C", [(1, 768), (197, 1000), (1999, 1000), (1999, 2048)])
def test_rmsnorm_sum_over_x(rows, C, wide):
    """The sum takes the place of x, and x may be the stream too; scales that lie anywhere, 16-byte aligned or not."""
    g, c = _g(), _g().ctx()
    rng = np.random.default_rng(rows + wide)
    x, res = norm_case(rng, rows, C, wide, wide, "ordinary")
    xs, gs = scale_channels(rng.uniform(0.3, 0.9, C)), scale_channels(rng.uniform(0.8, 1.1, C) * 32 * np.sqrt(C) / 2 ** 20)
    rs = Scale(*dyadic(0.96875))
    off = lambda a: torch.cat([torch.zeros(1, dtype=torch.from_numpy(a).dtype), torch.from_numpy(a)]).cuda()[1:]  # noqa: E731
    dx_scale, dgamma = (g.binding.DevScale.of(off(s.mult.astype(np.int32)), off(s.shift.astype(np.uint8))) for s in (xs, gs))
    assert dx_scale.mult_t.data_ptr() % 16 == 4
    drs = g.binding.DevScale(rs, "cuda")
    for same in (False, True):
        want, _, total = D.rmsnorm(x, (gs.mult, gs.shift), 20, (xs.mult, xs.shift), x if same else res, (rs.mult, rs.shift), wide == 1)
        dx = g.dev(x)
        dr = dx if same else g.dev(res)
        got = c.rmsnorm(dx, dgamma, x_scale=dx_scale, res=dr, res_scale=drs, sum_out=dx)
        g.assert_equal(g.host(got), want.astype(np.int8), f"out, {same}")
        g.assert_equal(g.host(dx), total.astype(x.dtype), f"sum, {same}")
        if not same:
            g.assert_equal(g.host(dr), res, "res")
