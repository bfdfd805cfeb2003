// Sizes and index arithmetic of the 4-bit key/value cache and of the attention over it (plain C++, so that the host can run it too).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define IVIT_KV4_FN __host__ __device__ __forceinline__
#else
#define IVIT_KV4_FN inline
#endif

namespace ivit {

// One (page, head) block: K codes [page][d/2], K steps [page][d/32], V codes [page][d/2], V steps [page].
IVIT_KV4_FN int64_t kv4_block_bytes(int d, int page) { return (int64_t)page * (d + d / 32 + 1); }
IVIT_KV4_FN int kv4_kcode(int d, int, int o) { return o * (d / 2); }
IVIT_KV4_FN int kv4_kstep(int d, int page, int o) { return page * (d / 2) + o * (d / 32); }
IVIT_KV4_FN int kv4_vcode(int d, int page, int o) { return page * (d / 2 + d / 32) + o * (d / 2); }
IVIT_KV4_FN int kv4_vstep(int d, int page, int o) { return page * (d + d / 32) + o; }

// What the lengths on the device allow a launch that was sized for max_q, max_len and `tokens` rows to touch.
struct Kv4Seq {
  int64_t q0;   // first row of Q and O
  int n;        // query tokens that are handled
  int nq;       // query tokens that the sequence has (saturated): places the last key
  int len;      // keys
  bool bad;
};
IVIT_KV4_FN Kv4Seq kv4_sequence(int q0, int q1, int len, int64_t tokens, int64_t max_q, int64_t max_len) {
  Kv4Seq s;
  s.bad = len < 0 || len > max_len;
  s.len = len < 0 ? 0 : (len > max_len ? (int)max_len : len);
  const int64_t nq = (int64_t)q1 - q0;
  int64_t n = nq < 0 ? 0 : nq;
  s.nq = (int)(n > 0x3fffffff ? 0x3fffffff : n);
  if (q0 < 0 || nq < 0 || nq > max_q || q1 > tokens) s.bad = true;
  if (n > max_q) n = max_q;
  if (q0 < 0) n = 0;
  else if (q0 + n > tokens) n = tokens > q0 ? tokens - q0 : 0;
  s.q0 = q0;
  s.n = (int)n;
  return s;
}
// Keys that query t sees: those up to its own, which is key len - nq + t.
IVIT_KV4_FN int kv4_seen(const Kv4Seq& s, int t) {
  const int v = s.len - s.nq + t + 1;
  return v < 0 ? 0 : (v > s.len ? s.len : v);
}

// A peer's maximum of a row, or 127 where the wait for it ran out and the place holds anything: the exponentials are looked up at maximum - score, and with
// a maximum that is no score's upper bound that would leave the table, and shared memory.  (The outputs are meaningless then, and the status says so.)
IVIT_KV4_FN int kv4_peer_top(bool arrived, int v) { return arrived ? v : 127; }

// ---- quotients of the attention ----

IVIT_KV4_FN int kv4_clz(unsigned long long n) {
#ifdef __CUDA_ARCH__
  return __clzll((long long)n);
#else
  return n ? __builtin_clzll(n) : 64;
#endif
}
IVIT_KV4_FN unsigned long long kv4_mul_hi(unsigned long long a, unsigned long long b) {
#ifdef __CUDA_ARCH__
  return __umul64hi(a, b);
#else
  return (unsigned long long)(((unsigned __int128)a * b) >> 64);
#endif
}
// About 2^64 / (den 2^up), up = leading zeros of den less 32 (den scaled to 32 bits with the upper one set; negative: cut): the reciprocal of
// its upper 16 bits by a 32-bit division (off by 2^-15), then one step of Newton's iteration (2^-29).  den < 2^43; 0 for den = 0.
// (A 64-bit division took 400 clocks more, with nothing beside it.)
IVIT_KV4_FN int up_of(unsigned long long den) { return kv4_clz(den) - 32; }
IVIT_KV4_FN unsigned long long recip_of(unsigned long long den) {
  if (!den) return 0;
  const int up = up_of(den);
  const unsigned d = (unsigned)(up >= 0 ? den << up : den >> -up);
  const unsigned v = 0xffffffffu / (d >> 16);                                       // about 2^48 / d, 17 bits
  const long long e = (long long)((1ull << 48) - (unsigned long long)v * d);        // of 2^48, at most 2^33 or so
  return ((unsigned long long)v << 16) + (unsigned long long)((e * (long long)v) >> 32);   // v 2^16 (1 + e / 2^48)
}

// floor(w / den) for |w| <= 2^24 den, den < 2^43 (0 for den = w = 0): the product with the reciprocal is off by less than 2^24 2^-28 and a
// unit, so by one at most, and multiplied back.  r = recip_of(den).
IVIT_KV4_FN int small_quotient(long long w, unsigned long long den, unsigned long long r) {
  const unsigned long long a = w < 0 ? 0ull - (unsigned long long)w : (unsigned long long)w;
  const int up = up_of(den);
  int q = (int)kv4_mul_hi(up >= 0 ? a << up : a >> -up, r);
  long long left = (long long)(a - (unsigned long long)(unsigned)q * den);
  if (left < 0) { --q; left += (long long)den; }
  if (left >= (long long)den && den) { ++q; left -= (long long)den; }
  return w < 0 ? -q - (left != 0) : q;
}

// Quotient of 0 <= n < 2^31 by a divisor that the host knows: the product's upper word, shifted (a multiplier of 32 bits, rounded up).
struct Kv4Div {
  unsigned d, m;
  int s;
  IVIT_KV4_FN int div(int n) const { return d == 1 ? n : (int)((unsigned)(((unsigned long long)(unsigned)n * m) >> 32) >> s); }
};
inline Kv4Div kv4_div(unsigned d) {
  int l = 0;
  while ((1u << l) < d) ++l;
  return Kv4Div{d, d > 1 ? (unsigned)(((1ull << (31 + l)) + d - 1) / d) : 0u, l - 1};
}

// ---- launch of the attention ----

constexpr int kKv4Block = 32;      // keys that a warp takes at a time
constexpr int kKv4Copies = 8;      // copies of the exponentials
constexpr int kKv4Blocks = 1024;   // most blocks of a CTA: a byte of codes times a byte of a weight, over 32768 keys, stays below 2^31
constexpr int kKv4Stages = 3;      // blocks that a warp holds: one that it works on, two on their way (us / with a fourth: 37 sequences of up to 7000 keys 32.5 /
                                   // 32.8, 2 of 20 000 16.0 / 16.6, pieces of prompts 63.1 / 63.2; 150 of 5000 89.2 / 87.8)
constexpr int kKv4Small = 3968;    // bytes of the rows' numbers
constexpr int kKv4SmemMax = 227 * 1024;

// Bytes of a row of scores in shared memory: 16 modulo 128, so that eight rows at the same keys lie in different banks.
IVIT_KV4_FN int kv4_score_ld(int blocks) { return (blocks * kKv4Block + 127) / 128 * 128 + 16; }
IVIT_KV4_FN int kv4_stage_bytes(int d) { return kKv4Block * (d / 2 + d / 32); }
// Words of a row of sums: 4 modulo 32, so that the lanes of a warp add to different banks.
IVIT_KV4_FN int kv4_sum_ld(int d) { return d + 4; }

struct Kv4Smem {
  int table, small, sums, peers, pages, ring, score, total;
};
// rows: query rows of a CTA (8 or 16); kept: those of them that some sequence can have, whose scores are kept; blocks: blocks of keys of a CTA;
// split: CTAs of a cluster; warps: of a CTA.
IVIT_KV4_FN Kv4Smem kv4_smem(int d, int rows, int kept, int page, int blocks, int split, int warps) {
  Kv4Smem m;
  m.table = 0;
  m.small = m.table + 256 * kKv4Copies * 4;
  m.sums = m.small + kKv4Small;
  m.peers = m.sums + 2 * rows * kv4_sum_ld(d) * 4;
  m.pages = m.peers + (split > 1 ? 16 * rows * (4 + 2 * 8) + (rows * d + 16) * 8 : 0);   // (see the kernel)
  m.ring = (m.pages + (blocks * kKv4Block / page + 2) * 8 + 127) / 128 * 128;
  // behind the passes the ring holds the shares of the weights
  const int ring = warps * kKv4Stages * kv4_stage_bytes(d), shares = rows * 256 * 4;
  m.score = m.ring + (ring > shares ? ring : shares);
  m.total = m.score + kept * kv4_score_ld(blocks);
  return m;
}

struct Kv4Plan {
  // query rows of a CTA, those with scores, CTAs of a cluster along the keys, blocks of each, warps, row tiles, bytes
  int rows, kept, split, blocks, warps, tiles, smem;
};
// room[c]: clusters of c CTAs, an SM for each, that the GPU runs at the same time (c <= 16).  The rules were drawn by measurement (us, of the two sides; 8
// heads of 128 unless noted):
//   16 query rows a CTA only where tiles of 8 would not run at once: 4 heads, 14 rows: 16 sequences of 3000 keys 15.0 / 13.5 with 8, 30 sequences 18.7 / 21.5
//   clusters from 24 blocks on, with 8 blocks a CTA at least: 2 sequences of 3000 keys 13.3 in one CTA each head / 8.1 in clusters, of 600 keys 6.9 / 7.5;
//   and no larger than run at once: one of 100 003 keys 33.0 in clusters of 10 / 46.8 in clusters of 16, which wait for one another
//   16 warps, alone on an SM, from 40 blocks a CTA on for each wave of CTAs (few of them: sequences are of uneven lengths, and the longest ends last), else
//   8, two CTAs on an SM, which overlap one another: 37 sequences of 7000 keys 32.5 / 42.9, of 2000 18.1 / 16.6; 150 of 3000 83 / 64
inline Kv4Plan kv4_plan(int d, int page, int64_t group, int64_t heads, int64_t seqs, int64_t max_q, int64_t max_len, int sms, const int* room) {
  Kv4Plan p;
  const int64_t all = (max_len + kKv4Block - 1) / kKv4Block, q_rows = max_q * group;
  for (p.rows = q_rows <= 8 || (q_rows + 7) / 8 * heads * seqs <= sms ? 8 : 16;; p.rows = 8) {
    p.tiles = (int)((q_rows + p.rows - 1) / p.rows);
    p.kept = (int)(q_rows < p.rows ? q_rows : p.rows);
    const int64_t ctas = (int64_t)p.tiles * heads * seqs;
    auto fits = [&]() {
      p.blocks = (int)((all + p.split - 1) / p.split);
      if (p.blocks < 1) p.blocks = 1;
      const int64_t waves = (ctas * p.split + sms - 1) / sms;
      for (p.warps = p.rows == 8 && p.blocks >= 40 * waves ? 16 : 8;; p.warps = 8) {
        p.smem = kv4_smem(d, p.rows, p.kept, page, p.blocks, p.split, p.warps).total;
        if (p.smem <= kKv4SmemMax && p.blocks <= kKv4Blocks) return true;
        if (p.warps == 8) return false;
      }
    };
    // (larger clusters than said only where the scores need the room)
    p.split = 16;
    while (p.split > 1 && (room[p.split] < ctas || all < 24 || all < 8 * p.split)) --p.split;
    bool ok = fits();
    while (!ok && p.split < 16) {
      ++p.split;
      ok = fits();
    }
    if (ok || p.rows == 8) return p;
  }
}

}  // namespace ivit
