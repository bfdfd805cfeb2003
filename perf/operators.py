"""Operators of an integer-only decoder, as cases that can be timed: a root-mean-square norm with the residual's addition, a
key/value cache held in 4 bits (append, attention over it, eviction from it by accumulated attention weight).

A case names an operator (`kind`) and its sizes.  Everything is integer arithmetic: every output is a whole number with one right
value, the bytes of the cache included (a code of 4 bits and its step are both whole numbers), so outputs are compared as they are.

`run` has each operator twice: as elementary torch operations (`own` false) and as the calls of this library (`own` true).
"""
import math

import numpy as np
import torch

own = False

M_LN = 20
I0, N = 17, 15               # ShiftExp: I0 = round(1 / S), pre-shift; the same as in this repository's attention workloads
TOP = I0 << N
Z = TOP.bit_length() - 8     # weights times the step of a value row are held in 16 bits
SINKS, RECENT = 4, 64


def listed():
    return [
        # one token of one sequence at the width of ViT-B: the smallest call, all latency
        dict(name="rms_1x768", kind="rmsnorm", rows=1, C=768, x32=False, h32=False, res=True, dynamic=False),
        # a decoding batch: Dense accumulators (int32) added to a wide stream, rows scaled one by one for what reads them
        dict(name="rms_64x4096_i32_rows", kind="rmsnorm", rows=64, C=4096, x32=True, h32=True, res=True, dynamic=True),
        # a long prompt, odd number of rows, int8 stream
        dict(name="rms_16383x2048", kind="rmsnorm", rows=16383, C=2048, x32=False, h32=False, res=True, dynamic=False),
        # one new token of each of 48 sequences goes into the cache
        dict(name="append_48", kind="append", tokens=48, heads=8, d=128, page=64),
        # a prompt goes into the cache
        dict(name="append_20011", kind="append", tokens=20011, heads=8, d=64, page=32),
        # one token of one sequence, the 197 tokens and 12 heads of ViT-B: latency
        dict(name="attend_b1_l197", kind="attend", B=1, Tq=1, L=197, hq=12, hk=12, d=64, page=32, weights=False),
        # decoding a ragged batch, four query heads on each key/value head, a sequence without keys among them
        dict(name="attend_b37_l7000", kind="attend", B=37, Tq=1, L=7000, hq=32, hk=8, d=128, page=64, weights=False),
        # one very long sequence: few rows, a long axis
        dict(name="attend_b1_l100003", kind="attend", B=1, Tq=1, L=100003, hq=32, hk=8, d=128, page=128, weights=False),
        # decoding that also accumulates the weights that eviction goes by
        dict(name="attend_b16_l3001_w", kind="attend", B=16, Tq=1, L=3001, hq=16, hk=8, d=64, page=64, weights=True),
        # pieces of prompts against what is in the cache already: many query rows, causal, ragged
        dict(name="attend_b5_t300_l2500", kind="attend", B=5, Tq=300, L=2500, hq=16, hk=4, d=128, page=64, weights=False),
        # eviction: a few short sequences, and a batch of long ones
        dict(name="evict_b3_l700", kind="evict", B=3, L=700, keep=333, hk=4, d=64, page=32),
        dict(name="evict_b12_l16001", kind="evict", B=12, L=16001, keep=4001, hk=8, d=128, page=64),
    ]


# ---- sizes drawn from the same ranges ----

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rmsnorm", "append", "attend", "attend", "attend", "evict"])
    top = [work(c) for c in listed() if c["kind"] == kind]
    while True:
        if kind == "rmsnorm":
            h32 = rng.random() < 0.4
            c = dict(kind=kind, rows=_log_int(rng, 1, 17000), C=4 * _log_int(rng, 8, 2048), x32=rng.random() < 0.4, h32=h32,
                     res=rng.random() < 0.8, dynamic=rng.random() < 0.4)
        elif kind == "append":
            c = dict(kind=kind, tokens=_log_int(rng, 1, 21000), heads=rng.randint(1, 16), d=rng.choice([64, 128]),
                     page=rng.choice([32, 64, 128, 256]))
        elif kind == "attend":
            hk = rng.randint(1, 12)
            c = dict(kind=kind, B=_log_int(rng, 1, 64), Tq=1 if rng.random() < 0.6 else _log_int(rng, 2, 400), L=_log_int(rng, 1, 100003),
                     hq=hk * rng.choice([1, 2, 3, 4, 7, 8]), hk=hk, d=rng.choice([64, 128]), page=rng.choice([32, 64, 128, 256]),
                     weights=rng.random() < 0.3)
            # the plain form holds every (query row, key) pair at once
            if c["B"] * c["hq"] * c["Tq"] * c["L"] > 6e7 or c["B"] * c["hk"] * c["L"] * c["d"] > 3e8:
                continue
        else:
            L = _log_int(rng, 200, 17000)
            c = dict(kind=kind, B=_log_int(rng, 1, 24), L=L, keep=rng.randint(SINKS + RECENT, max(SINKS + RECENT, (3 * L) // 4)),
                     hk=rng.randint(1, 12), d=rng.choice([64, 128]), page=rng.choice([32, 64, 128, 256]))
        w = work(c)
        if w["bytes"] <= max(t["bytes"] for t in top) and w["flops"] <= max(t["flops"] for t in top):
            return c


# ---- what follows from a case alone: lengths, pages ----

def _lengths(case):
    """(query tokens, keys) of every sequence: ragged; of three or more sequences one has no keys yet, so that no query of it sees any."""
    B, L, Tq = case["B"], case["L"], case.get("Tq", 0)
    lens = [L if b == 0 else 1 + (b * 7919 + 5) * 2654435761 % (1 << 32) * L // (1 << 32) for b in range(B)]
    if B >= 3 and case["kind"] == "attend":
        lens[1] = 0
    return [Tq if b == 0 else 1 + (b * 104729 + 3) * 2654435761 % (1 << 32) * Tq // (1 << 32) for b in range(B)], lens


def _block_bytes(case):
    """One page of one head: K codes, K steps, V codes, V steps."""
    return case["page"] * (case["d"] + case["d"] // 32 + 1)


def _pages(case):
    return -(-case["L"] // case["page"])


# ---- inputs ----

def _dyadic(ratio):
    s = 30 - math.floor(math.log2(ratio))
    m = int(round(ratio * 2.0 ** s))
    return (m, s) if m < 1 << 31 else (m >> 1, s - 1)


class _Make:
    """Device tensors made from the seed alone."""

    def __init__(self, seed):
        self.dev = torch.device("cuda", torch.cuda.current_device())
        self.g = torch.Generator(device=self.dev)
        self.g.manual_seed(int(seed) % (1 << 31))

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device=self.dev)

    def i8(self, std, *shape):
        """int8 rows, padded to a multiple of 16 bytes."""
        x = self.normal(*shape[:-1], -(-shape[-1] // 16) * 16).mul_(std).round_().clamp_(-128, 127).to(torch.int8)
        return x[..., :shape[-1]]

    def i32(self, std, *shape):
        return self.normal(*shape).mul_(std).round_().to(torch.int32)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=self.dev)

    def channel_scale(self, n, ratio):
        """One requantisation ratio per channel, spread by a tenth around `ratio`: (multipliers, shifts)."""
        ms = [_dyadic(ratio * (1.0 + 0.1 * v)) for v in self.normal(n).clamp_(-4, 4).tolist()]
        return (torch.tensor([m for m, _ in ms], dtype=torch.int32, device=self.dev),
                torch.tensor([s for _, s in ms], dtype=torch.uint8, device=self.dev))

    def cache(self, case, pages):
        """A pool with every row filled, as appended rows leave it; keys have a few channels of larger size, values do not."""
        hk, d, page = case["hk"], case["d"], case["page"]
        big = 1.0 + 2.0 * (torch.rand(hk, 1, d, generator=self.g, device=self.dev) < 0.06)
        pool = torch.empty((pages, hk, _block_bytes(case)), dtype=torch.uint8, device=self.dev)
        at = max(1, (1 << 24) // (hk * page * d))
        for p in range(0, pages, at):
            n = min(at, pages - p)
            k = (self.normal(n, hk, page, d) * (big * 24.0)).round_().clamp_(-128, 127).to(torch.int32)
            v = self.normal(n, hk, page, d).mul_(32.0).round_().clamp_(-128, 127).to(torch.int32)
            for part, rows in zip(_parts(pool[p:p + n], d, page), _quantise(k, v)):
                part.copy_(rows)
        return pool


def _handles():
    """The library, and the context that a program creates once and keeps."""
    from paper_2207_01405_b200 import binding
    key = (torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream)
    if key not in _contexts:
        _contexts[key] = binding.Context(key[0])
    return binding, _contexts[key]


_contexts = {}


def prepare(case, seed):
    mk, st, kind = _Make(seed), {"case": case}, case["kind"]
    if kind == "rmsnorm":
        rows, C = case["rows"], case["C"]
        st["x"] = mk.i32(20000.0, rows, C) if case["x32"] else mk.i8(32.0, rows, C)
        if case["res"]:
            target = 500.0 if case["h32"] else 10.0      # size of a branch in the units of the stream (ratios stay below 1)
            st["x_scale"] = mk.channel_scale(C, target / (20000.0 if case["x32"] else 1100.0))
            st["res"] = mk.i32(3000.0, rows, C) if case["h32"] else mk.i8(20.0, rows, C)
            st["res_scale"] = _dyadic(0.96875)
            st["sum"] = torch.zeros_like(st["res"]) if case["h32"] else mk.i8(0.0, rows, C)
        st["gamma"] = mk.channel_scale(C, 0.45 if case["dynamic"] else 32.0 * math.sqrt(C) / 2.0 ** M_LN)
        st["out"] = mk.i8(0.0, rows, C)
        st["row_max"] = torch.zeros(rows, dtype=torch.int32, device=mk.dev) if case["dynamic"] else None
    elif kind == "append":
        T, hk, d, page = case["tokens"], case["heads"], case["d"], case["page"]
        pages = -(-T // page) + 3
        qkv = mk.i8(32.0, T, 3 * hk * d)                 # the output of a QKV Dense: keys and values are column ranges
        st["k"], st["v"] = qkv[:, hk * d:2 * hk * d], qkv[:, 2 * hk * d:3 * hk * d]
        st["pool"] = torch.zeros((pages, hk, _block_bytes(case)), dtype=torch.uint8, device=mk.dev)
        st["slots"] = mk.perm(pages * page)[:T].contiguous()
        if T > 8:
            st["slots"][T // 3] = -1                     # a padded token
    elif kind == "attend":
        B, hq, hk, d, page = case["B"], case["hq"], case["hk"], case["d"], case["page"]
        tq, lens = _lengths(case)
        pages = B * _pages(case) + 2
        st["pool"] = mk.cache(case, pages)
        st["table"] = mk.perm(pages)[:B * _pages(case)].to(torch.int32).reshape(B, -1).contiguous()
        st["lens"] = torch.tensor(lens, dtype=torch.int32, device=mk.dev)
        st["q_start"] = torch.tensor([sum(tq[:b]) for b in range(B + 1)], dtype=torch.int32, device=mk.dev)
        st["q"] = mk.i8(32.0, sum(tq), hq * d)
        st["out"] = torch.zeros_like(st["q"])
        st["qk"] = _dyadic(25.0 / (8.0 * math.sqrt(d) * 32.0 * 27.0))
        st["pv"] = _dyadic(1.0 / 128.0)
        if case["weights"]:
            st["weights"] = torch.zeros((B, hk, _pages(case) * page), dtype=torch.int64, device=mk.dev)
    elif kind == "evict":
        B, hk, page = case["B"], case["hk"], case["page"]
        st["lens"] = torch.tensor(_lengths(case)[1], dtype=torch.int32, device=mk.dev)
        src, dst = _pages(case), -(-case["keep"] // page)
        st["pool"] = mk.cache(case, B * (src + dst))
        order = mk.perm(B * (src + dst)).to(torch.int32)
        st["table"], st["dst"] = order[:B * src].reshape(B, src).contiguous(), order[B * src:].reshape(B, dst).contiguous()
        # a few heavy keys, a long tail, and equal weights among the smallest
        w = (mk.normal(B, hk, src * page) * 3.0).exp_().mul_(2.0 ** 8).to(torch.int64)
        st["weights"] = torch.where(w < 64, w // 16, w << 6)
        st["weights_out"] = torch.empty_like(st["weights"][..., :dst * page])
        st["kept"] = torch.empty((B, hk, case["keep"]), dtype=torch.int32, device=mk.dev)
        st["new_lens"] = torch.empty(B, dtype=torch.int32, device=mk.dev)
    else:
        raise ValueError(kind)
    if own:   # what a program that uses the library keeps beside its tensors: its context, descriptions of its cache and scales
        binding, st["ctx"] = _handles()
        for name in ("x_scale", "res_scale", "gamma", "qk", "pv"):
            if name in st:
                st["dev_" + name] = binding.DevScale.of(*st[name])
        if kind != "rmsnorm":
            st["cache"] = binding.Kv4Cache(st["pool"], case["d"], case["page"])
            st["smax"] = binding.CExp(I0, N, 45, 8)
    return st


# ---- the operators ----

def run(st):
    c = st["case"]
    kind = c["kind"]
    if kind == "rmsnorm":
        if own:
            st["ctx"].rmsnorm(st["x"], st["dev_gamma"], x_scale=st.get("dev_x_scale"), res=st.get("res"),
                              res_scale=st.get("dev_res_scale"), M_ln=M_LN, sum_out=st.get("sum"), out=st["out"], row_max=st["row_max"])
            return [t for t in (st["out"], st["row_max"], st.get("sum")) if t is not None]
        return _plain_rmsnorm(st)
    if kind == "append":
        if own:
            st["ctx"].kv4_append(st["cache"], st["k"], st["v"], st["slots"])
            return st["pool"]
        return _plain_append(st)
    if kind == "attend":
        if own:
            st["ctx"].kv4_attention(st["cache"], st["q"], st["q_start"], st["lens"], st["table"], st["dev_qk"], st["smax"],
                                    st["dev_pv"], c["Tq"], c["L"], out=st["out"], weights=st.get("weights"))
            return [t for t in (st["out"], st.get("weights")) if t is not None]
        return _plain_attend(st)
    if own:
        st["ctx"].kv4_evict(st["cache"], st["weights"], st["lens"], st["table"], c["keep"], SINKS, RECENT, c["L"],
                            dst_table=st["dst"], weights_out=st["weights_out"], kept=st["kept"], new_lens=st["new_lens"])
        return st["kept"], st["new_lens"], st["weights_out"], st["pool"]
    return _plain_evict(st)


def _rq(a, mult, shift):
    """Round-half-up dyadic requantisation of int64 values; mult and shift per tensor (numbers) or per last-axis channel."""
    if torch.is_tensor(mult):
        mult, shift = mult.to(torch.int64), shift.to(torch.int64)
        return (a * mult + (torch.ones_like(shift) << (shift - 1))) >> shift
    return (a * mult + (1 << (shift - 1))) >> shift


def _bits(n):
    """Bit length of non-negative int64 values below 2^53."""
    return torch.frexp(n.double())[1].to(torch.int64)


def _plain_rmsnorm(st):
    x = st["x"].to(torch.int64)
    if "res" in st:
        h = _rq(x, *st["x_scale"]) + _rq(st["res"].to(torch.int64), *st["res_scale"])
        h = h.clamp_(-(1 << 20), 1 << 20) if st["res"].dtype == torch.int32 else h.clamp_(-128, 127)
    else:
        h = x.clamp(-(1 << 20), 1 << 20)
    V = (h * h).sum(-1, keepdim=True)
    sd = V.double().sqrt().to(torch.int64)
    sd = torch.where(sd * sd > V, sd - 1, sd)
    sd = torch.where((sd + 1) * (sd + 1) <= V, sd + 1, sd)
    e = _bits(sd).clamp(min=1)
    F = torch.where(sd > 0, (torch.ones_like(sd) << (M_LN + e)) // sd.clamp(min=1), 0)
    y = (h * F + (torch.ones_like(e) << (e - 1))) >> e
    z = _rq(y, *st["gamma"])
    outs = []
    if st["row_max"] is None:
        outs.append(z.clamp(-128, 127).to(torch.int8))
    else:
        A = z.abs().amax(-1, keepdim=True)
        a = _bits(A)
        R = torch.where(A > 0, (127 * torch.ones_like(A) << (23 + a)) // A.clamp(min=1), 0)
        outs += [((z * R + (torch.ones_like(a) << (22 + a))) >> (23 + a)).to(torch.int8), A.squeeze(-1).to(torch.int32)]
    if "res" in st:
        outs.append(h.to(st["res"].dtype))
    return outs


def _parts(pool, d, page):
    """Views of a pool [..., bytes]: K codes [..., page, d/2], K steps [..., page, d/32], V codes [..., page, d/2], V steps [..., page]."""
    a, b, c = page * d // 2, page * (d // 2 + d // 32), page * (d + d // 32)
    return (pool[..., :a].unflatten(-1, (page, d // 2)), pool[..., a:b].unflatten(-1, (page, d // 32)),
            pool[..., b:c].unflatten(-1, (page, d // 2)), pool[..., c:])


def _codes(x, step):
    """floor((16 x + step) / (2 step)), zero where the step is; x int32 [..., n], step [..., 1]."""
    return torch.where(step > 0, torch.div(16 * x + step, 2 * step.clamp(min=1), rounding_mode="floor"), 0)


def _quantise(k, v):
    """Rows [..., d] of int32 -> K codes, K steps, V codes, V steps as the cache's bytes hold them."""
    d = k.shape[-1]
    kg = k.unflatten(-1, (d // 32, 32))
    ks = torch.div(8 * kg.abs().amax(-1) + 6, 7, rounding_mode="floor")
    kc = (_codes(kg, ks[..., None]) + 8).unflatten(-1, (2, 4, 4))           # [..., group, half, t, i]
    kb = (kc[..., 0, :, :] | kc[..., 1, :, :] << 4).transpose(-3, -2).flatten(-3)   # byte 4 (groups t + group) + i
    vs = torch.div(8 * v.abs().amax(-1) + 6, 7, rounding_mode="floor")
    vc = (_codes(v, vs[..., None]) + 8).unflatten(-1, (2, d // 2))
    vb = vc[..., 0, :] | vc[..., 1, :] << 4
    return [t.to(torch.uint8) for t in (kb, ks, vb, vs)]


def _k_values(codes, steps, d):
    """K codes [..., d/2] and steps [..., d/32] -> eighths of a value [..., d], float64."""
    b = codes.unflatten(-1, (4, d // 32, 4)).transpose(-3, -2)               # [..., group, t, i]
    c = torch.stack((b & 15, b >> 4), -3).flatten(-3).to(torch.float64).sub_(8)
    return c.mul_(steps[..., None].to(torch.float64)).flatten(-2)


def _plain_append(st):
    c, pool, slots = st["case"], st["pool"], st["slots"]
    d, page, hk = c["d"], c["page"], c["heads"]
    t = (slots >= 0).nonzero().squeeze(-1)
    k, v = (st[n][t].to(torch.int32).unflatten(-1, (hk, d)) for n in ("k", "v"))
    p, o = slots[t] // page, slots[t] % page
    for part, rows in zip(_parts(pool, d, page), _quantise(k, v)):
        part[p[:, None], torch.arange(hk, device=p.device)[None], o[:, None]] = rows
    return pool


def _shift_exp(n):
    """ShiftExp(-n) for n >= 0, int64."""
    t = n + ((n + 1) >> 1) - ((n + 15) >> 4)
    q, r = t // I0, t % I0
    mant = I0 - ((r + 1) >> 1)
    return torch.where(q <= N, mant << (N - q).clamp(min=0), mant >> (q - N).clamp(min=0, max=62))


def _plain_attend(st):
    c = st["case"]
    B, Tq, hq, hk, d, page = c["B"], c["Tq"], c["hq"], c["hk"], c["d"], c["page"]
    G, dev = hq // hk, st["q"].device
    blocks = st["pool"][st["table"].long()].transpose(1, 2)                  # [B, hk, pages, bytes]
    kc, ks, vc, vs = (p.flatten(2, 3) for p in _parts(blocks, d, page))      # [B, hk, keys, ...]
    keys = kc.shape[2]
    start, lens = st["q_start"].long(), st["lens"].long()
    nq = start[1:] - start[:-1]
    t = torch.arange(Tq, device=dev)
    row = (start[:-1, None] + t).clamp(max=st["q"].shape[0] - 1)             # [B, Tq]
    q = st["q"][row].unflatten(-1, (hk, G, d)).permute(0, 2, 1, 3, 4).flatten(2, 3)   # [B, hk, Tq G, d]
    a = torch.matmul(q.to(torch.float64), _k_values(kc, ks, d).transpose(-1, -2)).to(torch.int64)
    s = _rq(a, *st["qk"]).clamp_(-128, 127)
    del a
    # query t of a sequence sees the keys up to its own place among the last nq keys
    last = (lens - nq)[:, None] + t                                          # [B, Tq]
    sees = torch.arange(keys, device=dev) <= last[..., None]
    sees = (sees & (t < nq[:, None])[..., None]).repeat_interleave(G, 1)[:, None]     # [B, 1, Tq G, keys]
    top = torch.where(sees, s, -1000).amax(-1, keepdim=True)
    e = torch.where(sees, _shift_exp((top - s).clamp_(min=0)), 0)
    del s
    den = e.sum(-1, keepdim=True)
    u = (e * vs.to(torch.int64)[:, :, None] + (1 << (Z - 1))) >> Z
    v = torch.cat(((vc & 15), (vc >> 4)), -1).to(torch.float64).sub_(8)
    num = torch.matmul(u.to(torch.float64), v).to(torch.int64)
    out = torch.where(den > 0, torch.div(num << (Z + 5), den.clamp(min=1), rounding_mode="floor"), 0)
    out = _rq(out, *st["pv"]).clamp_(-128, 127).to(torch.int8)
    out = out.unflatten(2, (Tq, G)).permute(0, 2, 1, 3, 4).flatten(2)        # [B, Tq, hq d]
    full = torch.zeros_like(st["q"])
    full[row[t < nq[:, None]]] = out[t < nq[:, None]]
    if "weights" not in st:
        return [full]
    st["weights"] += torch.where(den > 0, (e << 24) // den.clamp(min=1), 0).sum(2)
    return [full, st["weights"]]


def _plain_evict(st):
    c = st["case"]
    B, keep, hk, d, page = c["B"], c["keep"], c["hk"], c["d"], c["page"]
    w, lens = st["weights"], st["lens"].long()
    dev = w.device
    j = torch.arange(w.shape[-1], device=dev)
    held = (j < SINKS) | (j >= lens[:, None] - RECENT)
    order = torch.where(held[:, None], 1 << 62, w)
    order = torch.where((j < lens[:, None])[:, None], order, -1)
    pick = order.sort(dim=-1, descending=True, stable=True)[1][..., :keep]
    new = lens.clamp(max=keep)
    there = (torch.arange(keep, device=dev) < new[:, None])[:, None].expand(B, hk, keep)
    kept = torch.where(there, pick, w.shape[-1]).sort(-1)[0]
    at = kept.clamp(max=w.shape[-1] - 1)
    out = torch.zeros_like(st["weights_out"])
    out[..., :keep] = torch.where(there, w.gather(-1, at), 0)
    h = torch.arange(hk, device=dev)[None, :, None].expand(B, hk, keep)
    src = st["table"].long()[:, None].expand(B, hk, -1).gather(-1, at // page)
    k = torch.arange(keep, device=dev)
    dst = st["dst"].long()[:, None, k // page].expand(B, hk, keep)
    for part in _parts(st["pool"], d, page):
        part[dst[there], h[there], (k % page).expand(B, hk, keep)[there]] = part[src[there], h[there], (at % page)[there]]
    return torch.where(there, kept, -1).to(torch.int32), new.to(torch.int32), out, st["pool"]


# ---- the same from the definitions, number by number where it is quick, in numpy's 64-bit integers ----

def exact(case, seed):
    """What run() gives, for the smaller cases."""
    if work(case)["bytes"] > 3e6 or work(case)["flops"] > 3e7:
        return None
    st = prepare(case, seed)
    a = {k: v.cpu().numpy().astype(np.int64) for k, v in st.items() if torch.is_tensor(v)}
    if case["kind"] == "rmsnorm":
        scale = {n: [t.cpu().numpy().astype(np.int64) for t in st[n]] for n in ("x_scale", "gamma") if n in st}
        rows = [_exact_norm_row(case, a["x"][r], a["res"][r] if case["res"] else None, scale, st.get("res_scale")) for r in range(case["rows"])]
        outs = [np.array([r[0] for r in rows])]
        if case["dynamic"]:
            outs.append(np.array([r[1] for r in rows]))
        if case["res"]:
            outs.append(np.array([r[2] for r in rows]))
        return outs
    return _exact_attend(case, a, st) if case["kind"] == "attend" else _exact_append(case, a) if case["kind"] == "append" else _exact_evict(case, a)


def _exact_norm_row(case, x, res, scale, rs):
    lim = (-(1 << 20), 1 << 20) if case["h32"] or res is None else (-128, 127)
    h = [int(v) for v in x]
    if res is not None:
        m, s = scale["x_scale"]
        h = [((v * int(m[i]) + (1 << int(s[i]) - 1)) >> int(s[i])) + ((int(res[i]) * rs[0] + (1 << rs[1] - 1)) >> rs[1]) for i, v in enumerate(h)]
    h = [min(max(v, lim[0]), lim[1]) for v in h]
    sd = math.isqrt(sum(v * v for v in h))
    e = max(1, sd.bit_length())
    F = (1 << M_LN + e) // sd if sd else 0
    m, s = scale["gamma"]
    z = [(((v * F + (1 << e - 1)) >> e) * int(m[i]) + (1 << int(s[i]) - 1)) >> int(s[i]) for i, v in enumerate(h)]
    if not case["dynamic"]:
        return [min(max(v, -128), 127) for v in z], 0, h
    A = max(abs(v) for v in z)
    k = 23 + A.bit_length()
    R = (127 << k) // A if A else 0
    return [(v * R + (1 << k - 1)) >> k for v in z], A, h


def _places(case, o):
    """Byte ranges of row `o` of a page: K codes, K steps, V codes, V step."""
    d, page = case["d"], case["page"]
    at, out = 0, []
    for n in (d // 2, d // 32, d // 2, 1):
        out.append((at + o * n, at + (o + 1) * n))
        at += page * n
    return out


def _exact_append(case, a):
    pool, d = a["pool"].copy(), case["d"]
    for t, slot in enumerate(a["slots"]):
        for h in range(case["heads"]):
            if slot < 0:
                continue
            block, (kc, ks, vc, vs) = pool[slot // case["page"], h], _places(case, slot % case["page"])
            k, v = ([int(x) for x in a[n][t, h * d:(h + 1) * d]] for n in "kv")
            steps = [-(-8 * max(abs(x) for x in k[g:g + 32]) // 7) for g in range(0, d, 32)]
            code = [8 + ((16 * x + steps[c // 32]) // (2 * steps[c // 32]) if steps[c // 32] else 0) for c, x in enumerate(k)]
            for c in range(d):
                at = kc[0] + 4 * (d // 32 * (c % 16 // 4) + c // 32) + c % 4
                block[at] = code[c] | block[at] & 240 if c % 32 < 16 else code[c] << 4 | block[at] & 15
            block[ks[0]:ks[1]] = steps
            step = -(-8 * max(abs(x) for x in v) // 7)
            code = [8 + ((16 * x + step) // (2 * step) if step else 0) for x in v]
            block[vc[0]:vc[1]] = [code[c] | code[c + d // 2] << 4 for c in range(d // 2)]
            block[vs[0]] = step
    return pool


def _exact_evict(case, a):
    keep, page, pool = case["keep"], case["page"], a["pool"].copy()
    kept, out = np.full((case["B"], case["hk"], keep), -1), np.zeros(a["weights_out"].shape, np.int64)
    for b, L in enumerate(a["lens"]):
        for h in range(case["hk"]):
            free = [j for j in range(L) if SINKS <= j < L - RECENT]
            drop = set(sorted(free, key=lambda j: (a["weights"][b, h, j], -j))[:max(0, L - keep)])
            for n, j in enumerate(j for j in range(L) if j not in drop):
                kept[b, h, n], out[b, h, n] = j, a["weights"][b, h, j]
                for (s0, s1), (d0, d1) in zip(_places(case, j % page), _places(case, n % page)):
                    pool[a["dst"][b, n // page], h, d0:d1] = a["pool"][a["table"][b, j // page], h, s0:s1]
    return [kept, np.minimum(a["lens"], keep), out, pool]


def _exact_attend(case, a, st):
    hq, hk, d, page = case["hq"], case["hk"], case["d"], case["page"]
    out = np.zeros_like(a["q"])
    weights = np.zeros((case["B"], hk, a["table"].shape[1] * page), np.int64) if case["weights"] else None
    n = np.arange(256)
    t = n + ((n + 1) >> 1) - ((n + 15) >> 4)
    E = np.array([(I0 - ((r + 1) >> 1)) << (N - q) if q <= N else (I0 - ((r + 1) >> 1)) >> (q - N) for q, r in ((int(v) // I0, int(v) % I0) for v in t)])
    for b in range(case["B"]):
        L, q0, q1 = int(a["lens"][b]), int(a["q_start"][b]), int(a["q_start"][b + 1])
        for h in range(hk):
            K, V, vs = np.zeros((L, d), np.int64), np.zeros((L, d), np.int64), np.zeros(L, np.int64)
            for j in range(L):
                blk = a["pool"][a["table"][b, j // page], h]
                o = j % page
                kb, ks = blk[o * d // 2:(o + 1) * d // 2], blk[page * d // 2 + o * d // 32:page * d // 2 + (o + 1) * d // 32]
                vb = blk[page * (d // 2 + d // 32) + o * d // 2:page * (d // 2 + d // 32) + (o + 1) * d // 2]
                vs[j] = blk[page * (d + d // 32) + o]
                for g in range(d // 32):
                    byte = np.array([kb[4 * (d // 32 * w + g) + i] for w in range(4) for i in range(4)])
                    K[j, 32 * g:32 * g + 16], K[j, 32 * g + 16:32 * g + 32] = ((byte & 15) - 8) * ks[g], ((byte >> 4) - 8) * ks[g]
                V[j, :d // 2], V[j, d // 2:] = (vb & 15) - 8, (vb >> 4) - 8
            for r in range(q0, q1):
                seen = max(0, L - (q1 - q0) + (r - q0) + 1)
                for g in range(hq // hk):
                    if not seen:
                        continue
                    c0 = (h * (hq // hk) + g) * d
                    s = np.clip((K[:seen] @ a["q"][r, c0:c0 + d] * st["qk"][0] + (1 << st["qk"][1] - 1)) >> st["qk"][1], -128, 127)
                    e = E[s.max() - s]
                    den = int(e.sum())
                    u = (e * vs[:seen] + (1 << Z - 1)) >> Z
                    tt = (u @ V[:seen] << Z + 5) // den
                    out[r, c0:c0 + d] = np.clip((tt * st["pv"][0] + (1 << st["pv"][1] - 1)) >> st["pv"][1], -128, 127)
                    if weights is not None:
                        weights[b, h, :seen] += (e << 24) // den
    return [out] if weights is None else [out, weights]


# ---- what a pass cannot do without ----

def work(case):
    kind = case["kind"]
    if kind == "rmsnorm":
        n, C = case["rows"] * case["C"], case["C"]
        x, h = 4 if case["x32"] else 1, 4 if case["h32"] else 1
        return {"bytes": float(n * (x + (2 * h if case["res"] else 0) + 1) + C * (10 if case["res"] else 5) + (4 * case["rows"] if case["dynamic"] else 0)),
                "flops": 16.0 * n}
    if kind == "append":
        n, d = case["tokens"] * case["heads"], case["d"]
        return {"bytes": float(n * (2 * d + d + d // 32 + 1) + 8 * case["tokens"]), "flops": 10.0 * n * d}
    d, page, hk = case["d"], case["page"], case["hk"]
    tq, lens = _lengths(case)
    row = d + d // 32 + 1
    if kind == "attend":
        hq = case["hq"]
        pairs = sum(sum(min(L, max(0, L - t + i + 1)) for i in range(t)) for t, L in zip(tq, lens)) * hq
        return {"bytes": float(sum(lens) * hk * (row + (16 if case["weights"] else 0)) + 2 * sum(tq) * hq * d + 4 * sum(-(-L // page) for L in lens)),
                "flops": 4.0 * d * pairs + hq * d}
    kept = sum(min(L, case["keep"]) for L in lens)
    return {"bytes": float(hk * (8 * sum(lens) + kept * (2 * row + 12))), "flops": 8.0 * hk * sum(lens)}
