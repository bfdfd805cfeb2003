"""CPU side of the decoder operators: the reference pinned against floating point and closed forms, the scalars that host and device
share, and every refusal of the entry points (arguments are checked before anything of the context or the device is touched)."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from ivit_inputs import Scale
from ivit_inputs.gen import dyadic
from oracle import api as O
from oracle import decoder as D

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---- the reference ----

def test_reference_uses_the_library_s_exponential_and_rounding():
    rng = np.random.default_rng(0)
    for I0, N in ((17, 15), (1, 14), (32767, 9), (255, 0)):
        for n in list(range(256)):
            assert int(D.shiftexp(n, I0, N)) == O.shiftexp(-n, I0, N)
    for a, m, s in zip(rng.integers(-2 ** 31, 2 ** 31, 500), rng.integers(1, 2 ** 31, 500), rng.integers(31, 63, 500)):
        assert int(D.rq(int(a), int(m), int(s))) == O.rq(int(a), int(m), int(s))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 256])
def test_cache_bytes_round_trip(d, page):
    rng = np.random.default_rng(d + page)
    raw = rng.integers(0, 256, (3, 2, page * (d + d // 32 + 1))).astype(np.uint8)
    assert np.array_equal(D.Cache.of_bytes(raw, d, page).to_bytes(), raw)


def test_quantisation_error_is_half_a_step():
    """code step / 8 is off by at most half a step (exactly: 16 |8 x - code step| <= 8 step 2), and a code never passes 7."""
    rng = np.random.default_rng(1)
    for std in (0.5, 3, 30, 200):
        x = np.clip(np.rint(rng.standard_normal((4000, 32)) * std), -128, 127).astype(np.int64)
        code, step = D._quantise(x)
        assert np.abs(code).max() <= 7 and step.max() <= 147 and step.min() >= 0
        assert (2 * np.abs(8 * x - code * step) <= step).all()


def test_attention_reference_against_floating_point():
    """Against exp and an exact division on the cache's own values.  ShiftExp's weights are p_j (1 + x_j) before they are normalised, |x_j| <= x
    (read off the table of all differences of scores), which moves an average by at most x / (1 - x) sum p_j |v_j - average|; u_j is off by half
    a unit of 2^z, which moves it by at most 7 2^(z-1) / 8 for each key over den; the floor of t by 1/256; the last rounding by 1/2."""
    rng = np.random.default_rng(2)
    d, page, L, I0, N = 64, 32, 500, 64, 15
    ref = D.Cache(16, 1, d, page)
    k = np.clip(np.rint(rng.standard_normal((L, d)) * 32), -128, 127).astype(np.int8)
    v = np.clip(np.rint(rng.standard_normal((L, d)) * 32), -128, 127).astype(np.int8)
    ref.append(k, v, np.arange(L))
    q = np.clip(np.rint(rng.standard_normal((1, d)) * 32), -128, 127).astype(np.int8)
    ratio, gain = 20.0 / (8 * math.sqrt(d) * 32 * 32), 127 / 128
    out, w = D.attention(ref, q, 1, [0, 1], [L], np.arange(16)[None], dyadic(ratio), I0, N, dyadic(gain / 256), np.zeros((1, d)),
                         np.zeros((1, 1, L), np.int64))
    K = (ref.kc.reshape(-1, d) * np.repeat(ref.ks.reshape(-1, d // 32), 32, -1))[:L] / 8
    V = (ref.vc.reshape(-1, d) * ref.vs.reshape(-1, 1))[:L] / 8
    s = np.clip(np.floor(K @ q[0] * 8 * ratio + 0.5), -128, 127)
    n = np.arange(int(s.max() - s.min()) + 1)
    x = np.abs(D.shiftexp(n, I0, N) / (I0 << N) / np.exp(-n / I0) - 1).max()
    p = np.exp((s - s.max()) / I0)
    den = p.sum() * (1 - x) * (I0 << N)
    p /= p.sum()
    z = (I0 << N).bit_length() - 8
    avg = p @ V
    tol = 0.5 + gain * (x / (1 - x) * (p[:, None] * np.abs(V - avg)).sum(0) + 7 * 2 ** (z - 1) / 8 * L / den + 1 / 256) + 1e-6
    assert (np.abs(out[0] - avg * gain) <= tol).all()
    assert (np.abs(w[0, 0] / 2 ** 24 - p) <= 2 * x / (1 - x) * p + 2.0 ** -24).all()
    assert 2 ** 24 - L <= w.sum() <= 2 ** 24


def test_rmsnorm_reference_against_floating_point():
    rng = np.random.default_rng(3)
    C_, M = 777 // 4 * 4, 20
    for std, wide in ((20, False), (3000, True), (200000, True)):
        h = np.rint(rng.standard_normal((6, C_)) * std).astype(np.int64)
        ratio = 30 * math.sqrt(C_) / 2 ** M
        out, _, _ = D.rmsnorm(h, dyadic(ratio), M)
        hc = np.clip(h, -2 ** 20, 2 ** 20)
        want = 30 * hc / np.sqrt((hc.astype(float) ** 2).mean(-1, keepdims=True))
        # half a unit of rounding, and the floor of the root: at most one part in sd, |value| <= 128
        assert np.abs(out - np.clip(want, -128, 127)).max() <= 0.5 + 129 / (std * math.sqrt(C_) * 0.9) + 0.01
        out, top, _ = D.rmsnorm(h, dyadic(0.5), M, dynamic=True)
        z = out * top[:, None] / 127
        assert np.abs(out).max(-1).tolist() == [127] * 6 and np.abs(z - want / 30 * 2 ** M / math.sqrt(C_) / 2).max() <= top.max() / 254 + 0.002 * top.max()


# ---- scalars of a row, compiled for the host ----

def test_row_scalars_on_the_host(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text('#include "rms_scalars.cuh"\n'
                   'extern "C" unsigned root(unsigned long long n) { return ivit::isqrt56(n); }\n'
                   'extern "C" void row(unsigned long long V, int M, int* F, int* e) { auto k = ivit::rms_row(V, M); *F = k.F; *e = k.e; }\n'
                   'extern "C" void scale(int A, int* R, int* sh) { ivit::rms_row_scale(A, *R, *sh); }\n')
    so = tmp_path / "t.so"
    subprocess.run(["g++", "-O2", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2207_01405_b200", "csrc"), "-o", str(so), str(src)], check=True)
    L = C.CDLL(str(so))
    L.root.argtypes, L.root.restype = [C.c_ulonglong], C.c_uint
    L.row.argtypes = [C.c_ulonglong, C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int)]
    L.scale.argtypes = [C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int)]
    rng = np.random.default_rng(4)
    ns = [n for b in range(56) for n in ((1 << b) - 1, 1 << b, (1 << b) + 1)] + [2 ** 56 - 1]
    ns += [r * r + o for r in rng.integers(2 ** 12, 2 ** 28 - 1, 20000).tolist() for o in (-1, 0, 1)]
    ns += [int(2 ** x) for x in rng.uniform(0, 56, 50000)]
    for n in ns:
        if 0 <= n < 2 ** 56:
            assert L.root(n) == math.isqrt(n), n
    a, b = C.c_int(), C.c_int()
    for n in ns[:2000]:
        for M in (8, 20, 22):
            L.row(n, M, C.byref(a), C.byref(b))
            sd = math.isqrt(n)
            assert (a.value, b.value) == (((1 << (M + sd.bit_length())) // sd, sd.bit_length()) if sd else (0, 0))
    for A in list(range(1, 3000)) + rng.integers(1, 2 ** 23, 3000).tolist() + [2 ** 22, 2 ** 22 + 1]:
        L.scale(A, C.byref(a), C.byref(b))
        assert b.value == 23 + A.bit_length() and a.value == (127 << b.value) // A and a.value < 2 ** 31
    L.scale(0, C.byref(a), C.byref(b))
    assert a.value == 0


# ---- index arithmetic of the attention, compiled for the host ----

@pytest.fixture(scope="module")
def layout(tmp_path_factory):
    src = tmp_path_factory.mktemp("layout") / "t.cpp"
    src.write_text('#include "kv4_layout.cuh"\nusing namespace ivit;\nextern "C" {\n'
                   'void plan(int d, int page, int64_t g, int64_t h, int64_t s, int64_t q, int64_t l, int sms, const int* room, int* o) {\n'
                   '  Kv4Plan p = kv4_plan(d, page, g, h, s, q, l, sms, room); Kv4Smem m = kv4_smem(d, p.rows, p.kept, page, p.blocks, p.split, p.warps);\n'
                   '  int v[] = {p.rows, p.split, p.blocks, p.tiles, p.smem, m.table, m.small, m.sums, m.peers, m.pages, m.ring, m.score, kv4_score_ld(p.blocks), kv4_sum_ld(d), p.kept, kKv4Stages, p.warps};\n'
                   '  for (int i = 0; i < 17; ++i) o[i] = v[i]; }\n'
                   'void seq(int q0, int q1, int len, int64_t tok, int64_t mq, int64_t ml, int64_t* o) {\n'
                   '  Kv4Seq s = kv4_sequence(q0, q1, len, tok, mq, ml); o[0] = s.q0; o[1] = s.n; o[2] = s.nq; o[3] = s.len; o[4] = s.bad; }\n'
                   'int seen(int q0, int q1, int len, int64_t tok, int64_t mq, int64_t ml, int t) { return kv4_seen(kv4_sequence(q0, q1, len, tok, mq, ml), t); }\n'
                   'void places(int d, int page, int o, int64_t* v) { v[0] = kv4_kcode(d, page, o); v[1] = kv4_kstep(d, page, o); v[2] = kv4_vcode(d, page, o);\n'
                   '  v[3] = kv4_vstep(d, page, o); v[4] = kv4_block_bytes(d, page); }\n'
                   'int quotient(int64_t w, uint64_t den) { return small_quotient(w, den, recip_of(den)); }\n}\n')
    so = src.with_suffix(".so")
    subprocess.run(["g++", "-O2", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2207_01405_b200", "csrc"), "-o", str(so), str(src)], check=True)
    L = C.CDLL(str(so))
    i64 = C.c_int64
    L.plan.argtypes = [C.c_int, C.c_int, i64, i64, i64, i64, i64, C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int)]
    L.seq.argtypes = [C.c_int, C.c_int, C.c_int, i64, i64, i64, C.POINTER(i64)]
    L.seen.argtypes = [C.c_int, C.c_int, C.c_int, i64, i64, i64, C.c_int]
    L.quotient.argtypes = [i64, C.c_uint64]
    L.places.argtypes = [C.c_int, C.c_int, C.c_int, C.POINTER(i64)]
    return L


def test_every_launch_fits(layout):
    """The plan of a launch covers every key and query row, and the parts of shared memory follow one another inside the limit."""
    rng = np.random.default_rng(6)
    o = (C.c_int * 17)()
    rooms = [[0, 148, 74, 45, 33, 26, 22, 15, 15, 15, 11, 7, 7, 7, 7, 7, 7], [0, 148] + [0] * 15, [148] * 17]
    room = (C.c_int * 17)()
    lens = [0, 1, 31, 32, 33, 256, 257, 1000, 4096, 12288, 12289, 24577, 65536, 100003, 131073, 196607, 196608]
    for d in (64, 128):
        for page in (32, 256):
            for L in lens + rng.integers(1, 196609, 30).tolist():
                for g, h, s, q in ((1, 1, 1, 1), (4, 8, 1, 1), (8, 8, 64, 1), (9, 2, 3, 1), (16, 1, 1, 1), (17, 1, 1, 1), (4, 8, 5, 300), (1, 65535, 65535, 1),
                                   (7, 3, 2, 1 << 24)):
                    room[:] = rooms[(L + g) % 3]
                    layout.plan(d, page, g, h, s, q, L, 148, room, o)
                    rows, split, blocks, tiles, smem, table, small, sums, peers, pages, ring, score, ld, sum_ld, kept, stages, warps = list(o)
                    assert rows in (8, 16) and 1 <= split <= 16 and smem <= 227 * 1024
                    assert tiles * rows >= q * g > (tiles - 1) * rows
                    assert split * blocks * 32 >= L and blocks >= 1
                    assert small - table >= 256 * 8 * 4 and sums - small >= 4 * 320 + 8 * 322 and peers - sums >= 2 * rows * sum_ld * 4 and pages >= peers and ring - pages >= 8 * (blocks * 32 // page + 2)
                    assert stages >= 2 and (warps == 8 or (warps == 16 and rows == 8)) and score - ring >= max(warps * stages * 32 * (d // 2 + d // 32), rows * 1024) and sum_ld >= d
                    assert split == 1 or (pages - peers >= 16 * rows * 20 + 8 * (rows * d + 16) and peers % 8 == 0 and -(-rows * d // split) * split <= rows * d + 16)
                    assert ld >= blocks * 32 and ld % 128 == 16 and smem >= score + kept * ld and 1 <= kept == min(rows, q * g)
                    assert ring % 128 == 0 and score % 16 == 0 and pages % 16 == 0 and small % 16 == 0
                    # eight rows, four words each, at the same keys: 32 banks
                    assert len({(r * ld // 4 + t) % 32 for r in range(8) for t in range(4)}) == 32
                    assert len({(2 * t * ld // 4 + n) % 32 for t in range(4) for n in range(8)}) == 32
                    assert len({(2 * t * sum_ld + n) % 32 for t in range(4) for n in range(8)}) == 32
                    # sums of a CTA stay below 2^31: a byte of codes times a byte of a weight
                    assert 255 * 255 * 32 * blocks < 2 ** 31


def test_quotients(layout):
    """floor(w / den) at and around every multiple that matters, over the whole range of denominators."""
    rng = np.random.default_rng(7)
    assert layout.quotient(0, 0) == 0
    for n in range(60000):
        b = int(rng.integers(1, 43))
        den = max(1, [int(rng.integers(1 << (b - 1), 1 << b)), (1 << b) - 1, (1 << b) - 2, 1 << (b - 1), (1 << (b - 1)) + 1][n % 5])
        q = int(rng.integers(0, 1 << int(rng.integers(1, 25))))
        for w in (q * den, q * den + den - 1, q * den + int(rng.integers(0, den))):
            if w < 1 << 62 and w <= den << 24:
                assert layout.quotient(w, den) == w // den and layout.quotient(-w, den) == -w // den, (w, den)


def test_what_a_sequence_may_touch(layout):
    o = (C.c_int64 * 5)()
    ends = [-2 ** 31, -1, 0, 1, 5, 7, 8, 100, 2 ** 30, 2 ** 31 - 1]
    for q0 in ends:
        for q1 in ends:
            for ln in ends:
                for tok, mq, ml in ((8, 3, 100), (1, 1, 1), (100, 100, 196608)):
                    layout.seq(q0, q1, ln, tok, mq, ml, o)
                    s, n, nq, L, bad = list(o)
                    assert 0 <= n <= mq and 0 <= L <= ml and (n == 0 or (s >= 0 and s + n <= tok))
                    assert bool(bad) == (not (0 <= q0 <= q1 <= tok and q1 - q0 <= mq and 0 <= ln <= ml))
                    if not bad:
                        assert (n, nq, L, s) == (q1 - q0, q1 - q0, ln, q0)
                    last = -1
                    for t in range(min(n, 10)):
                        seen = layout.seen(q0, q1, ln, tok, mq, ml, t)
                        assert 0 <= seen <= L and seen >= last
                        last = seen
                        if not bad:
                            assert seen == max(0, ln - (q1 - q0) + t + 1)


def test_places_in_a_block(layout):
    v = (C.c_int64 * 5)()
    for d in (64, 128):
        for page in (32, 64, 128, 256):
            used = np.zeros(page * (d + d // 32 + 1), int)
            for o in range(page):
                layout.places(d, page, o, v)
                for at, n in zip(v, (d // 2, d // 32, d // 2, 1)):
                    used[at:at + n] += 1
                assert v[4] == len(used) and v[4] % 16 == 0
            assert (used == 1).all()


# ---- refusals ----

@pytest.fixture(scope="module")
def lib():
    from paper_2207_01405_b200 import binding, build
    build.build()
    return binding


def test_call_descriptions_have_the_header_s_layout(lib, tmp_path):
    """Every field of the structures of ivit.h lies where the binding packs it."""
    src = tmp_path / "t.c"
    fields = {"rmsnorm": "x ldx res ldres sum ldsum out ldout row_max rows C x_scale res_scale gamma_scale x_dtype res_dtype M_ln",
              "kv4_attention": "Q ldq O ldo q_start lens table ldtable weights ldw q_heads tokens seqs max_q max_len qk_scale pv_scale smax",
              "kv4_evict": "weights ldw weights_out ldw_out lens new_lens table ldtable dst_table ld_dst kept seqs max_len keep sinks recent"}
    body = "".join(f'  printf("%zu ", sizeof(ivit_{n}_params));\n' + "".join(f'  printf("%zu ", offsetof(ivit_{n}_params, {f}));\n' for f in fs.split()) +
                   '  printf("\\n");\n' for n, fs in fields.items())
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ivit.h"\nint main(void) {\n' + body + "  return 0;\n}\n")
    exe = tmp_path / "t"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [[int(v) for v in line.split()] for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines()]
    scale, eight = 24, 8
    want = []
    for n, fs in fields.items():
        at, offs = 0, []
        for f in fs.split():
            offs.append(at)
            at += scale if f.endswith("_scale") else 16 if f == "smax" else 4 if f in ("x_dtype", "res_dtype", "M_ln") else eight
        want.append([-(-at // 8) * 8] + offs)
    assert got == want
    assert [lib._RMSNORM.size, lib._ATTENTION.size, lib._EVICT.size] == [w[0] for w in want]


CTX = C.create_string_buffer(8192)          # never looked at: every call here is refused, or has nothing to do
AT = 1 << 20                                # an aligned address that is never read


def rms(b, **k):
    v = dict(ctx=C.addressof(CTX), x=AT, xd=0, ldx=64, xs=b.CScale(None, None, 2 ** 30, 33), res=None, rd=0, ldr=0, rs=b.CScale(None, None, 2 ** 30, 31),
             gs=b.CScale(None, None, 2 ** 30, 35), M=20, sum=None, lds=0, out=AT, ldo=64, rm=None, rows=1, C=64)
    v.update(k)
    f = lambda s: (s.mult_c or 0, s.shift_c or 0, s.mult, s.shift)  # noqa: E731
    z = lambda n: v[n] or 0  # noqa: E731
    d = b._RMSNORM.pack(z("x"), v["ldx"], z("res"), v["ldr"], z("sum"), v["lds"], z("out"), v["ldo"], z("rm"), v["rows"], v["C"], *f(v["xs"]), *f(v["rs"]),
                        *f(v["gs"]), v["xd"], v["rd"], v["M"])
    return b.load_library().ivit_rmsnorm(v["ctx"], d)


def test_rmsnorm_refusals(lib):
    b = lib
    bad = b.CScale(None, None, 0, 33)
    chan = b.CScale(AT, AT, 0, 0)
    for code, k in ((-1, dict(ctx=None)), (-1, dict(x=None)), (-1, dict(out=None)), (-1, dict(rows=-1)), (-1, dict(C=0)), (-1, dict(xd=2)),
                    (-1, dict(sum=AT, lds=64)), (-1, dict(res=AT, rd=5, ldr=64)), (-4, dict(C=66)), (-4, dict(C=16388, ldx=16400, ldo=16400)),
                    (-3, dict(M=7)), (-3, dict(M=23)), (-1, dict(ldx=48)), (-1, dict(ldo=48)), (-1, dict(res=AT, ldr=48)),
                    (-1, dict(res=AT, ldr=64, sum=AT, lds=32)), (-2, dict(x=AT + 4)), (-2, dict(ldx=68)), (-2, dict(out=AT + 1)), (-2, dict(ldo=72)),
                    (-2, dict(xd=1, ldx=66)), (-2, dict(res=AT, ldr=65)), (-2, dict(res=AT, ldr=64, sum=AT, lds=66)), (-2, dict(rm=AT + 2)),
                    (-3, dict(gs=bad)), (-3, dict(res=AT, ldr=64, xs=bad)), (-3, dict(res=AT, ldr=64, rs=bad)), (-3, dict(res=AT, ldr=64, rs=chan)),
                    (-3, dict(gs=b.CScale(AT, None, 0, 0))), (-3, dict(gs=b.CScale(None, None, 5, 63))), (-3, dict(gs=b.CScale(None, None, 5, 30))),
                    (-2, dict(gs=b.CScale(AT + 2, AT, 0, 0)))):
        assert rms(b, **k) == code, k


def cache(b, **k):
    v = dict(data=AT, pages=4, heads=2, d=64, page=32)
    v.update(k)
    return b.CKv4(v["data"], v["pages"], v["heads"], v["d"], v["page"])


BAD_CACHES = [(-1, dict(data=None)), (-1, dict(pages=0)), (-1, dict(heads=0)), (-4, dict(d=32)), (-4, dict(d=96)), (-4, dict(page=48)),
              (-4, dict(page=16)), (-4, dict(page=512)), (-4, dict(pages=1 << 31)), (-4, dict(heads=65536)), (-2, dict(data=AT + 8))]


def test_cache_bytes(lib):
    L = lib.load_library()
    for d in (64, 128):
        for page in (32, 64, 128, 256):
            assert L.ivit_kv4_cache_bytes(C.byref(cache(lib, d=d, page=page, pages=5, heads=3))) == 15 * page * (d + d // 32 + 1)
    assert L.ivit_kv4_cache_bytes(C.byref(cache(lib, data=None, pages=1 << 30, heads=65535, d=128, page=256))) == (65535 << 30) * 256 * 133
    assert L.ivit_kv4_cache_bytes(None) == 0
    for code, k in BAD_CACHES:
        if code != -2 and "data" not in k:
            assert L.ivit_kv4_cache_bytes(C.byref(cache(lib, **k))) == 0


def append(b, c=None, **k):
    v = dict(ctx=C.addressof(CTX), K=AT, ldk=128, V=AT, ldv=128, slots=AT, tokens=1)
    v.update(k)
    return b.load_library().ivit_kv4_append(v["ctx"], C.byref(c or cache(b)), v["K"], v["ldk"], v["V"], v["ldv"], v["slots"], v["tokens"])


def test_append_refusals(lib):
    for code, k in BAD_CACHES:
        assert append(lib, cache(lib, **k)) == code, k
    for code, k in ((-1, dict(ctx=None)), (-1, dict(K=None)), (-1, dict(V=None)), (-1, dict(slots=None)), (-1, dict(tokens=-1)), (-1, dict(ldk=112)),
                    (-1, dict(ldv=112)), (-2, dict(K=AT + 4)), (-2, dict(V=AT + 8)), (-2, dict(ldk=136)), (-2, dict(ldv=129)), (-2, dict(slots=AT + 4)),
                    (-4, dict(tokens=(1 << 40) + 1))):
        assert append(lib, **k) == code, k


def attend(b, c=None, **k):
    one = b.CScale(None, None, 2 ** 30, 40)
    v = dict(ctx=C.addressof(CTX), Q=AT, ldq=256, qh=4, tokens=3, qs=AT, lens=AT, table=AT, ldt=4, qk=one, p=b.CExp(17, 15, 45, 8), pv=one, O=2 * AT,
             ldo=256, w=None, ldw=0, seqs=2, mq=2, ml=100)
    v.update(k)
    f = lambda s: (s.mult_c or 0, s.shift_c or 0, s.mult, s.shift)  # noqa: E731
    z = lambda n: v[n] or 0  # noqa: E731
    d = b._ATTENTION.pack(z("Q"), v["ldq"], z("O"), v["ldo"], z("qs"), z("lens"), z("table"), v["ldt"], z("w"), v["ldw"], v["qh"], v["tokens"], v["seqs"],
                          v["mq"], v["ml"], *f(v["qk"]), *f(v["pv"]), v["p"].I0, v["p"].N, v["p"].M, v["p"].k_out)
    return b.load_library().ivit_kv4_attention(v["ctx"], C.byref(c or cache(b)), d)


def test_attention_refusals(lib):
    b = lib
    chan, bad = b.CScale(AT, AT, 0, 0), b.CScale(None, None, -4, 40)
    for code, k in BAD_CACHES:
        assert attend(b, cache(b, **k)) == code, k
    for code, k in ((-1, dict(ctx=None)), (-1, dict(Q=None)), (-1, dict(O=None)), (-1, dict(O=AT)), (-1, dict(qs=None)), (-1, dict(lens=None)),
                    (-1, dict(table=None)), (-1, dict(tokens=-1)), (-1, dict(seqs=-1)), (-1, dict(mq=-1)), (-1, dict(ml=-1)), (-1, dict(qh=3)),
                    (-1, dict(qh=0)), (-1, dict(qh=1)), (-1, dict(ldq=240)), (-1, dict(ldo=240)), (-1, dict(ldt=3)), (-1, dict(w=AT, ldw=99)),
                    (-4, dict(ml=196609, ldt=10000)), (-4, dict(seqs=65536)), (-4, dict(mq=1 << 24)), (-4, dict(tokens=1 << 31)),
                    (-4, dict(qh=65536, ldq=65536 * 64, ldo=65536 * 64)), (-2, dict(Q=AT + 8)), (-2, dict(O=2 * AT + 1)), (-2, dict(ldq=264)),
                    (-2, dict(ldo=257)), (-2, dict(qs=AT + 2)), (-2, dict(lens=AT + 1)), (-2, dict(table=AT + 3)), (-2, dict(w=AT + 4, ldw=100)),
                    (-3, dict(qk=chan)), (-3, dict(pv=chan)), (-3, dict(qk=bad)), (-3, dict(pv=bad)), (-3, dict(p=b.CExp(0, 15, 45, 8))),
                    (-3, dict(p=b.CExp(17, 25, 45, 8))), (-3, dict(p=b.CExp(17, -1, 45, 8))), (-3, dict(p=b.CExp(17, 15, 44, 8))),
                    (-3, dict(p=b.CExp(1, 13, 45, 8))), (-3, dict(p=b.CExp(1, 24, 45, 8))), (-3, dict(p=b.CExp(32768, 9, 45, 8))),
                    (-3, dict(p=b.CExp(32769, 1, 45, 8)))):
        assert attend(b, **k) == code, k
    for k in (dict(tokens=0, Q=None, O=None), dict(seqs=0, lens=None, table=None, qs=None), dict(mq=0)):
        assert attend(b, **k) == 0, k


def evict(b, c=None, **k):
    v = dict(ctx=C.addressof(CTX), w=AT, ldw=100, lens=AT, table=AT, ldt=4, dst=2 * AT, ldd=2, wo=2 * AT, ldwo=64, kept=AT, new=AT, seqs=1, ml=100,
             keep=50, sinks=4, recent=20)
    v.update(k)
    z = lambda n: v[n] or 0  # noqa: E731
    d = b._EVICT.pack(z("w"), v["ldw"], z("wo"), v["ldwo"], z("lens"), z("new"), z("table"), v["ldt"], z("dst"), v["ldd"], z("kept"), v["seqs"], v["ml"],
                      v["keep"], v["sinks"], v["recent"])
    return b.load_library().ivit_kv4_evict(v["ctx"], C.byref(c or cache(b)), d)


def test_evict_refusals(lib):
    b = lib
    for code, k in BAD_CACHES:
        assert evict(b, cache(b, **k)) == code, k
    for code, k in ((-1, dict(ctx=None)), *((-1, {n: None}) for n in ("w", "lens", "table", "dst", "wo", "kept", "new")), (-1, dict(seqs=-1)),
                    (-1, dict(ml=-1)), (-1, dict(keep=0)), (-1, dict(sinks=-1)), (-1, dict(recent=-1)), (-1, dict(sinks=31)), (-1, dict(sinks=51, recent=0)),
                    (-1, dict(recent=47)), (-1, dict(recent=2 ** 63 - 1)), (-1, dict(ldw=99)), (-1, dict(ldwo=49)), (-1, dict(ldt=3)), (-1, dict(ldd=1)),
                    (-1, dict(dst=AT)), (-1, dict(wo=AT)), (-4, dict(seqs=65536)), (-4, dict(ml=1 << 31, ldw=1 << 31, ldt=1 << 30)),
                    (-2, dict(w=AT + 4)), (-2, dict(wo=AT + 4)), (-2, dict(lens=AT + 2)), (-2, dict(table=AT + 2)), (-2, dict(dst=AT + 2)),
                    (-2, dict(kept=AT + 2)), (-2, dict(new=AT + 2))):
        assert evict(b, **k) == code, k


def test_evict_refuses_what_its_indices_do_not_hold(lib):
    """Indices are 32 bits and run up to a turn of all threads past the last key: 2^30 keys are the limit, of max_len and of keep."""
    for k in (dict(ml=(1 << 30) + 1), dict(ml=(1 << 31) - 1), dict(keep=(1 << 30) + 1, ml=100), dict(keep=(1 << 31) - 1)):
        assert evict(lib, **{**dict(ldw=1 << 31, ldt=1 << 30, ldwo=1 << 31, ldd=1 << 30), **k}) == -4, k
    assert evict(lib, ml=1 << 30, keep=1 << 30, ldw=1 << 31, ldt=1 << 30, ldwo=1 << 31, ldd=1 << 30, seqs=0) == 0


def test_rmsnorm_refuses_a_sum_that_runs_over_its_own_stream(lib):
    """sum == res with other leading dimensions: a row of the sum would lie on rows of res that are still to be read."""
    for lds, ldr in ((64, 80), (80, 64)):
        assert rms(lib, res=AT, ldr=ldr, sum=AT, lds=lds, rows=4) == -1
    assert rms(lib, res=AT, ldr=80, sum=AT, lds=80, rows=0) == 0


def test_scales_that_are_not_on_the_device_are_refused(lib):
    """An array of multipliers in host memory would be read by the GPU as an address of its own."""
    mult, shift = torch.full((64,), 2 ** 30, dtype=torch.int32), torch.full((64,), 35, dtype=torch.uint8)
    for m, s in ((mult, shift), (mult, 35), (mult.long(), shift), (mult, shift[:32])):
        with pytest.raises(ValueError):
            lib.DevScale.of(m, s)
    c = object.__new__(lib.Context)          # (no device, no library call: only the check)
    c.index, c.device = 0, "cuda:0"
    scale = lib.DevScale(Scale(mult.numpy(), shift.numpy()), "cpu")
    for n in (64, 32):
        with pytest.raises(ValueError):
            c._fields(scale, n)
    c.index = -1
    assert c._fields(scale, 64) == scale.fields and c._fields(lib.DevScale.of(2 ** 30, 35), 7) == (0, 0, 2 ** 30, 35)
    c.h = None


def test_evict_of_no_sequences_to_other_pages(lib):
    """Tensors without elements have no address: that both are null does not make the call one in place."""
    none = dict(seqs=0, w=None, wo=None, lens=None, table=None, dst=None, kept=None, new=None)
    assert evict(lib, **none) == 0
    assert evict(lib, **none, ldt=100, ldd=2, ldw=100, ldwo=50) == 0
    assert evict(lib, **none, keep=0) == -1


def test_evict_without_keys_needs_no_tables(lib):
    """max_len = 0: there is nothing to read or to move, and tables and weights without columns have no address.  What is written has to be there."""
    none = dict(seqs=0, ml=0, w=None, table=None, dst=None)
    assert evict(lib, **none) == 0
    for n in ("lens", "wo", "kept", "new"):
        assert evict(lib, **{**none, "seqs": 3, n: None}) == -1, n
    for n in ("w", "table", "dst"):
        assert evict(lib, **{n: None}) == -1, n


def test_rmsnorm_refuses_a_sum_that_runs_over_x(lib):
    """sum == x with another leading dimension or type: words of it would lie on values of x that other threads have still to read."""
    for k in (dict(lds=80, ldx=64), dict(lds=64, ldx=80), dict(xd=1, lds=64), dict(rd=1, lds=64)):
        assert rms(lib, **{**dict(res=2 * AT, ldr=80, sum=AT, rows=4), **k}) == -1, k
    for k in (dict(xd=0, rd=0), dict(xd=1, rd=1), dict(xd=1, lds=80)):       # (the same place, or no rows)
        assert rms(lib, **{**dict(res=2 * AT, ldr=80, sum=AT, lds=64, rows=0), **k}) == 0, k


@pytest.mark.parametrize("L,far", [(300, 187), (3000, 187), (30000, 187), (30000, 120), (30000, 0)])
def test_what_the_weights_16_bits_cost(L, far):
    """A key's weight u is off by half a unit of 2^z at most, so by 7 2^z / 16 in the numerator's units of a value: over all keys that are seen the output is within
    7 L 2^z / (16 den) of a value's unit of the one with weights that are not rounded (t: and its floor, 1/256).  Where one key holds the weight, the others
    far below it, nearly all of that comes about: den is top, more than 2^(z+7), and the tail of a long row is rounded away from the numerator alone."""
    rng = np.random.default_rng(L + far)
    I0, N, d = 17, 15, 64
    z = (I0 << N).bit_length() - 8
    vs, vc = np.full(L, 100), np.full((L, d), 7)
    vc[:, d // 2:] = rng.integers(-7, 8, (L, d // 2))
    diff = np.full(L, far)
    diff[0] = 0
    vs[0], vc[0] = 100, 0
    e = D.shiftexp(diff, I0, N)
    den = int(e.sum())
    u = (e * vs + (1 << (z - 1))) >> z
    t = np.array([(int(v) << (z + 5)) // den for v in u @ vc]) / 256
    exact = (e * vs) @ vc / (8 * den)
    bound = 7 * L * 2 ** z / (16 * den)
    assert (np.abs(t - exact) <= bound + 1 / 256 + 1e-9).all()
    assert bound <= L / 292                                          # (den >= top >= 2^(z+7))
    if far == 187:                                                   # 100 e < 2^(z-1): the whole tail is gone, and it would have counted
        assert (u[1:] == 0).all() and (t == 0).all() and exact[0] > 0.45 * bound
    if far == 0:
        assert np.abs(t - exact).max() <= 7 / 2048 + 1 / 256


def test_a_maximum_that_did_not_arrive_stays_inside_the_table(tmp_path):
    """Behind a wait that ran out a peer's maximum is whatever shared memory held.  The row's maximum over sixteen of them, some of them there, looks every
    score up inside the 256 exponentials all the same."""
    src = tmp_path / "t.cpp"
    src.write_text('#include <climits>\n#include "kv4_layout.cuh"\nusing namespace ivit;\nint main() {\n'
                   '  const int junk[] = {INT_MIN, -100000, -129, -128, 0, 127, 128, 65536, INT_MAX};\n'
                   '  for (int v : junk)\n    for (int there = -128; there < 128; ++there)\n      for (int n = 0; n < 16; ++n) {\n'
                   '        int top = -128;\n        for (int k = 0; k < 16; ++k) {\n          const int t = k < n ? kv4_peer_top(true, there) : kv4_peer_top(false, v);\n'
                   '          top = t > top ? t : top;\n        }\n'
                   '        for (int score = -128; score < 128; ++score)\n          if (top - score < 0 || top - score > 255) return 1;\n      }\n'
                   '  for (int v = -128; v < 128; ++v)\n    if (kv4_peer_top(true, v) != v) return 2;\n  return 0;\n}\n')
    exe = tmp_path / "t"
    subprocess.run(["g++", "-O2", "-I", os.path.join(ROOT, "paper_2207_01405_b200", "csrc"), "-o", str(exe), str(src)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
