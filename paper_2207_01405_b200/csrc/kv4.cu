// A key/value cache held in 4 bits: append to it, eviction from it (sm_100a).  Layout: ivit_kv4_cache in ivit.h.
#include "common.cuh"
#include "kv4_layout.cuh"

namespace ivit {

__device__ __forceinline__ void report(int* status, int code) { *(volatile int*)status = code; }

struct Cache {
  uint8_t* data;
  int64_t pages;
  int heads, page, page_log, block_bytes;
  __device__ __forceinline__ uint8_t* block(int pg, int h) const { return data + ((int64_t)pg * heads + h) * block_bytes; }
};

static Cache to_dev(const ivit_kv4_cache* c) {
  int lg = 0;
  while ((1 << lg) < c->page) ++lg;
  return Cache{c->data, c->pages, (int)c->heads, (int)c->page, lg, (int)kv4_block_bytes((int)c->d, (int)c->page)};
}

// ---------------------------------------------------------------- append

__device__ __forceinline__ int signed_byte(uint32_t w, int b) {
  int d;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(d) : "r"(w), "r"(0x8880 + 0x1111 * b));
  return d;
}
__device__ __forceinline__ unsigned max_s16x2(unsigned a, unsigned b) {
  unsigned d;
  asm("max.s16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ unsigned min_s16x2(unsigned a, unsigned b) {
  unsigned d;
  asm("min.s16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ unsigned two_bytes(uint32_t w, int from) {   // bytes from, from + 1, sign-extended to 16 bits
  unsigned d;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(d) : "r"(w), "r"(from ? 0xb3a2 : 0x9180));
  return d;
}
// Largest magnitude of sixteen int8, two 16-bit values at a time: the larger of the maximum and of the minimum turned round.
__device__ __forceinline__ int top_of(const uint32_t (&w)[4]) {
  unsigned hi = two_bytes(w[0], 0), lo = hi;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const unsigned v = two_bytes(w[i >> 1], 2 * (i & 1));
    hi = max_s16x2(hi, v);
    lo = min_s16x2(lo, v);
  }
  return max(max((int)(short)hi, (int)hi >> 16), -min((int)(short)lo, (int)lo >> 16));
}
// ceil(8 top / 7), top <= 128.
__device__ __forceinline__ int step_of(int top) { return (8 * top + 6) / 7; }
// code + 8 of four values, one in each byte: floor((16 x + 17 step) / (2 step)), the numerator below 4548 and the quotient below 16, by a
// product with r = floor(2^23 / step) + 1 (off by less than 4548 / 2^24 < 1 / (2 step)), whose upper byte is the quotient.  r = 0 and
// eight in the end where the step is 0.
__device__ __forceinline__ uint32_t codes_of(uint32_t w, int step, unsigned r) {
  const unsigned m = 16u * r, c0 = 17u * (unsigned)step * r;   // (the sum is below 2^29, whatever its parts are modulo 2^32)
  unsigned p[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) p[b] = (unsigned)signed_byte(w, b) * m + c0;
  const uint32_t c = __byte_perm(__byte_perm(p[0], p[1], 0x0073), __byte_perm(p[2], p[3], 0x0073), 0x5410);
  return step ? c : 0x08080808u;
}

// Codes of sixteen values of this lane and of the lane `other` away, low and high halves of the same bytes: words 0 and 1 of the four go to the
// lane with the low halves, 2 and 3 to the one with the high ones.
__device__ __forceinline__ uint2 join(const uint32_t (&c)[4], bool high, int other) {
  const uint32_t x = __shfl_xor_sync(~0u, high ? c[0] : c[2], other), y = __shfl_xor_sync(~0u, high ? c[1] : c[3], other);
  return high ? make_uint2(x | c[2] << 4, y | c[3] << 4) : make_uint2(c[0] | x << 4, c[1] | y << 4);
}

// D / 16 lanes take a row of one token and head: sixteen channels each of K and of V.  The lanes with a byte's low and high halves are
// neighbours in K, D / 32 apart in V.  What bounds it is the issue of instructions: 20 011 tokens x 8 heads of 64 9.7 us (31 MB would take 4.8), of 128 17.4;
// with eight channels a lane, and so twice the reductions, steps and addresses, 12.5 and 22.9.  Two rows for each lane were no gain (9.7 and 16.6, a call of
// 48 tokens 1.9 -> 2.5).
template <int D>
__global__ void __launch_bounds__(256) kv4_append_kernel(const Cache c, const int8_t* __restrict__ K, int64_t ldk, const int8_t* __restrict__ V,
                                                         int64_t ldv, const int64_t* __restrict__ slots, unsigned rows, Kv4Div by_heads, int* status) {
  constexpr int L = D / 16;                      // lanes of a row
  __shared__ unsigned recip[256];
  if (threadIdx.x < 148) recip[threadIdx.x] = threadIdx.x ? (1u << 23) / threadIdx.x + 1u : 0u;
  pdl_wait();
  pdl_trigger();
  const int l = threadIdx.x & (L - 1);
  const unsigned mine = blockIdx.x * (256 / L) + threadIdx.x / L, r = min(mine, rows - 1), t = (unsigned)by_heads.div((int)r);
  const int h = (int)(r - t * by_heads.d);
  const uint4 k = *reinterpret_cast<const uint4*>(K + t * ldk + (h * D + 16 * l)), v = *reinterpret_cast<const uint4*>(V + t * ldv + (h * D + 16 * l));
  const long long slot = mine < rows ? slots[t] : -1;
  __syncthreads();
  uint32_t kw[4] = {k.x, k.y, k.z, k.w}, vw[4] = {v.x, v.y, v.z, v.w};
  int kt = top_of(kw), vt = top_of(vw);
  kt = max(kt, __shfl_xor_sync(~0u, kt, 1));
#pragma unroll
  for (int o = 1; o < L; o <<= 1) vt = max(vt, __shfl_xor_sync(~0u, vt, o));
  const int ks = step_of(kt), vs = step_of(vt);
  const unsigned kr = recip[ks], vr = recip[vs];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    kw[i] = codes_of(kw[i], ks, kr);
    vw[i] = codes_of(vw[i], vs, vr);
  }
  const bool k_high = l & 1, v_high = l >= L / 2;
  const uint2 kc = join(kw, k_high, 1), vc = join(vw, v_high, L / 2);
  if (slot < 0) return;
  if (slot >> c.page_log >= c.pages) {
    if (l == 0) report(status, IVIT_ERR_RANGE);
    return;
  }
  uint8_t* p = c.block((int)(slot >> c.page_log), h);
  const int o = (int)slot & (c.page - 1), g = l >> 1;
  uint32_t* dst = reinterpret_cast<uint32_t*>(p + kv4_kcode(D, c.page, o)) + D / 32 * (k_high ? 2 : 0) + g;   // words 0 and 1, or 2 and 3, of group g
  dst[0] = kc.x;
  dst[D / 32] = kc.y;
  *reinterpret_cast<uint2*>(p + kv4_vcode(D, c.page, o) + 16 * (l & (L / 2 - 1)) + (v_high ? 8 : 0)) = vc;
  if (!k_high) p[kv4_kstep(D, c.page, o) + g] = (uint8_t)ks;
  if (l == 1) p[kv4_vstep(D, c.page, o)] = (uint8_t)vs;
}

int launch_kv4_append(ivit_ctx* ctx, const ivit_kv4_cache* cache, const int8_t* K, int64_t ldk, const int8_t* V, int64_t ldv,
                      const int64_t* slots, int64_t tokens) {
  if (tokens == 0) return IVIT_OK;
  LaunchScope ls(ctx, KIND_MOVE, (double)tokens * cache->heads * (3 * cache->d + cache->d / 32 + 1));
  const unsigned rows = (unsigned)(tokens * cache->heads);
  auto go = [&](auto k, unsigned per) {
    launch_k(k, (rows + per - 1) / per, 256, 0, ctx->stream, to_dev(cache), K, ldk, V, ldv, slots, rows, kv4_div((unsigned)cache->heads), ctx->status_dev);
  };
  if (cache->d == 128) go(kv4_append_kernel<128>, 32);
  else go(kv4_append_kernel<64>, 64);
  return ls.done();
}

// ---------------------------------------------------------------- eviction

struct EvictArgs {
  Cache c;
  const int64_t* w; int64_t ldw;
  const int32_t *lens, *table; int64_t ldtable;
  const int32_t* dst; int64_t ld_dst;
  int64_t* w_out; int64_t ldw_out;
  int32_t *kept, *new_lens;
  int max_len, keep, sinks, recent;
  int* status;
};

__device__ __forceinline__ unsigned long long order_key(long long w) { return (unsigned long long)w ^ (1ull << 63); }

__device__ __forceinline__ int evict_len(const EvictArgs& a, int b) {
  const int len = a.lens[b];
  if (len < 0 || len > a.max_len) {
    if (threadIdx.x == 0) report(a.status, IVIT_ERR_RANGE);
    return max(0, min(len, a.max_len));
  }
  return len;
}

// First digit of a weight's order: its bit length and the five bits behind the leading one.  Accumulated weights are spread over many powers
// of two: digits of that kind leave few keys in the one that holds the threshold, and few lanes that count in the same place.
constexpr int kDigits = 2048;
__device__ __forceinline__ int first_digit(unsigned long long k) {
  const int e = 64 - __clzll((long long)k);
  return e <= 5 ? (int)k : ((e - 5) << 5) + (int)((k >> (e - 6)) & 31);
}

// One CTA for each (sequence, head), its warps on runs of keys one behind the other (kRegs: of at most 512 keys, held in registers; else
// read again in each pass).  Finds the smallest weight that stays, then lists the keys in order:
//   1. counts of the first digits, and the digit in which `need` of the largest are reached;
//   2. the keys of that digit: one value (small weights; all equal) needs no more, up to 1024 are ranked against one another, more are told apart byte by byte;
//   3. each warp counts what stays of its run, and writes it behind what stays of the runs in front.
// 12 sequences x 8 heads of 16 001 keys: 20 us, of which the weights' 12.3 MB would be 2; with 96 CTAs it is their passes, one behind the other, that
// count.  Reading the keys again in each pass takes 19 us more (41.2 / 60.1 for the whole call), for 4000 keys 3 us (13.6 / 16.8).
template <bool kRegs>
__global__ void __launch_bounds__(1024) kv4_select_kernel(const EvictArgs a) {
  constexpr int kKeys = 16;
  __shared__ unsigned hist[kDigits];
  __shared__ unsigned long long list[1024];
  __shared__ unsigned count, need_s, digit_s, sums[32], ties_s[32];
  __shared__ unsigned long long prefix_s, low_s, high_s;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.x, b = blockIdx.y;
  const int len = evict_len(a, b);
  const int64_t bh = (int64_t)b * a.c.heads + h;
  int32_t* kept = a.kept + bh * a.keep;
  if (len <= a.keep) {
    for (int j = tid; j < a.keep; j += 1024) kept[j] = j < len ? j : -1;
    return;
  }
  const int64_t* w = a.w + bh * a.ldw;
  const int lo = a.sinks, hi = len - a.recent;               // candidates
  unsigned need = (unsigned)(a.keep - a.sinks - a.recent);   // of them
  const int run = (len + 1023) / 1024 * 32, j0 = min(len, warp * run), j1 = min(len, j0 + run);
  unsigned long long keys[kRegs ? kKeys : 1];
  if (kRegs) {
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int j = j0 + 32 * i + lane;
      keys[kRegs ? i : 0] = j < j1 ? order_key(w[j]) : 0;
    }
  }
  // f(index, key, there) for the warp's keys, 32 at a time
  auto each = [&](auto f) {
    if (kRegs) {
#pragma unroll
      for (int i = 0; i < kKeys; ++i)
        if (j0 + 32 * i < j1) f(j0 + 32 * i + lane, keys[kRegs ? i : 0], j0 + 32 * i + lane < j1);
    } else {
      for (int jb = j0; jb < j1; jb += 32) f(jb + lane, jb + lane < j1 ? order_key(w[jb + lane]) : 0ull, jb + lane < j1);
    }
  };
  unsigned long long prefix = ~0ull;   // need == 0: nothing is above, nothing equal stays
  if (need > 0) {
    // (order_key flips the sign: zero is 2^63.  The digits are those of the weight itself, negative ones all in the first.)
    auto digit = [&](unsigned long long k) { return k >> 63 ? first_digit(k & ~(1ull << 63)) : 0; };
    for (int i = tid; i < kDigits; i += 1024) hist[i] = 0;
    if (tid == 0) count = 0, low_s = ~0ull, high_s = 0;
    bool negative = false;
    __syncthreads();
    unsigned none = 0;   // digit 0 (weights of zero are common): counted lane by lane
    each([&](int j, unsigned long long k, bool) {
      if (j >= lo && j < hi) {
        const int g = digit(k);
        if (g) atomicAdd(&hist[g], 1u);
        else ++none;
        negative |= !(k >> 63);
      }
    });
    negative = __syncthreads_or(negative) != 0;
    none = __reduce_add_sync(~0u, none);
    if (lane == 0 && none) atomicAdd(&hist[0], none);
    __syncthreads();
    {  // thread t has digits 2047 - 2 t and 2046 - 2 t: sums over what is above
      const unsigned x = hist[kDigits - 1 - 2 * tid], y = hist[kDigits - 2 - 2 * tid];
      unsigned s = x + y;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned v = __shfl_up_sync(~0u, s, o);
        if (lane >= o) s += v;
      }
      if (lane == 31) sums[warp] = s;
      __syncthreads();
      unsigned front = lane < warp ? sums[lane] : 0;
      front = __reduce_add_sync(~0u, front) + s - x - y;      // above this thread's two digits
      if (front < need && need <= front + x) { digit_s = kDigits - 1 - 2 * tid; need_s = need - front; }
      else if (front + x < need && need <= front + x + y) { digit_s = kDigits - 2 - 2 * tid; need_s = need - front - x; }
    }
    __syncthreads();
    const int at = (int)digit_s;
    need = need_s;
    const unsigned in_digit = hist[at];
    if (at < 64 && !(at == 0 && negative)) {
      prefix = order_key(at);              // (digits below 64 are the weights themselves)
    } else if (in_digit <= 1024) {
      each([&](int j, unsigned long long k, bool) {
        if (j >= lo && j < hi && digit(k) == at) list[atomicAdd(&count, 1u)] = k;
      });
      __syncthreads();
      if (tid < (int)in_digit) {
        const unsigned long long k = list[tid];
        unsigned above = 0, same = 0;
        for (unsigned i = 0; i < in_digit; ++i) {
          above += list[i] > k;
          same += list[i] == k;
        }
        if (above < need && need <= above + same) { prefix_s = k; need_s = need - above; }   // (equal keys all say the same)
      }
      __syncthreads();
      prefix = prefix_s;
      need = need_s;
    } else {
      // (all of them equal: the one value)
      unsigned long long low = ~0ull, high = 0;
      each([&](int j, unsigned long long k, bool) {
        if (j >= lo && j < hi && digit(k) == at) low = min(low, k), high = max(high, k);
      });
      if (low <= high) atomicMin(&low_s, low), atomicMax(&high_s, high);
      __syncthreads();
      prefix = low_s;
      for (int shift = low_s == high_s ? -8 : 56; shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        each([&](int j, unsigned long long k, bool) {
          const bool in = j >= lo && j < hi && digit(k) == at && (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8)));
          const unsigned v = in ? (unsigned)(k >> shift) & 255u : 256u, peers = __match_any_sync(~0u, v);   // (many are equal: one addition for all of a warp)
          if (in && lane == __ffs(peers) - 1) atomicAdd(&hist[v], (unsigned)__popc(peers));
        });
        __syncthreads();
        if (tid == 0) {
          unsigned n = need;
          int v = 255;
          while (v > 0 && hist[v] < n) n -= hist[v--];
          prefix_s = (shift == 56 ? 0ull : prefix) | (unsigned long long)v << shift;
          need_s = n;
        }
        __syncthreads();
        prefix = prefix_s;
        need = need_s;
      }
    }
  }
  // ---- weights above `prefix` stay, and the first `need` of those equal to it
  unsigned above = 0, ties = 0, up_bits = 0, tie_bits = 0;   // (of this lane's keys, in order: one bit of each word for each turn)
  int turn = 0;
  each([&](int j, unsigned long long k, bool there) {
    const bool up = there && (j < lo || j >= hi || k > prefix), tie = there && !up && k == prefix;
    if (kRegs) up_bits |= (unsigned)up << turn, tie_bits |= (unsigned)tie << turn, ++turn;
    above += up;
    ties += tie;
  });
  above = __reduce_add_sync(~0u, above);
  ties = __reduce_add_sync(~0u, ties);
  __syncthreads();   // (sums was read above)
  if (lane == 0) { sums[warp] = above; ties_s[warp] = ties; }
  __syncthreads();
  unsigned at_above = __reduce_add_sync(~0u, lane < warp ? sums[lane] : 0), at_ties = __reduce_add_sync(~0u, lane < warp ? ties_s[lane] : 0);
  const unsigned below = (1u << lane) - 1;
  turn = 0;
  each([&](int j, unsigned long long k, bool there) {
    bool up, tie;
    if (kRegs) {
      up = up_bits >> turn & 1;
      tie = tie_bits >> turn & 1;
      ++turn;
    } else {
      up = there && (j < lo || j >= hi || k > prefix);
      tie = there && !up && k == prefix;
    }
    const unsigned mu = __ballot_sync(~0u, up), mt = __ballot_sync(~0u, tie);
    const unsigned t = at_ties + __popc(mt & below);
    if (up || (tie && t < need)) kept[at_above + __popc(mu & below) + min(t, need)] = j;
    at_above += __popc(mu);
    at_ties += __popc(mt);
  });
}

// Moves the rows that stay, 16 bytes of K and of V to a thread.  kOrdered (in place): one CTA for each (sequence, head), group of rows behind
// group of rows, each loaded before any of it is stored; rows that are read later lie behind those that are written.  Else the groups of rows are
// shared out.  Bound by the latency of three dependent loads (index, page, row), hence the rows that a thread has
// under way: 12 sequences x 8 heads, 4001 rows of 16 001, 27 us alone, 0.45 of the DRAM's peak.
template <int D, bool kOrdered>
__global__ void __launch_bounds__(kOrdered ? 512 : 256) kv4_compact_kernel(const EvictArgs a) {
  constexpr int kParts = D / 32, U = 4;                            // threads of a row; rows of a thread
  constexpr int kThreads = kOrdered ? 512 : 256, kRows = kThreads / kParts;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, part = tid % kParts;
  const int h = blockIdx.y, b = blockIdx.z;
  const int n = min(evict_len(a, b), a.keep);
  const int64_t bh = (int64_t)b * a.c.heads + h;
  const int32_t* kept = a.kept + bh * a.keep;
  const int32_t *from = a.table + b * a.ldtable, *to = a.dst + b * a.ld_dst;
  const int64_t *w_in = a.w + bh * a.ldw;
  int64_t* w_out = a.w_out + bh * a.ldw_out;
  const int kstep = kv4_kstep(D, a.c.page, 0), vcode = kv4_vcode(D, a.c.page, 0), vstep = kv4_vstep(D, a.c.page, 0);
  for (int i0 = blockIdx.x * (kRows * U); i0 < n; i0 += gridDim.x * (kRows * U)) {
    uint4 k[U], v[U];
    uint32_t st[U];
    int64_t w[U];
    int j[U], sp[U], dp[U];
    // (each of the three loads for all U rows at once)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * kRows + tid / kParts, n - 1);
      j[u] = kept[i];
      dp[u] = to[i >> a.c.page_log];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) sp[u] = from[j[u] >> a.c.page_log];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kRows + tid / kParts, o = j[u] & (a.c.page - 1);
      const bool there = i < n && sp[u] >= 0 && sp[u] < a.c.pages && dp[u] >= 0 && dp[u] < a.c.pages;
      const uint8_t* s = a.c.block(there ? sp[u] : 0, h);
      if (!there) dp[u] = -1;
      k[u] = v[u] = make_uint4(0, 0, 0, 0);
      st[u] = 0;
      w[u] = 0;
      if (there) {
        k[u] = *reinterpret_cast<const uint4*>(s + o * (D / 2) + 16 * part);
        v[u] = *reinterpret_cast<const uint4*>(s + vcode + o * (D / 2) + 16 * part);
        if (part == 0) st[u] = D == 128 ? *reinterpret_cast<const uint32_t*>(s + kstep + o * 4) : *reinterpret_cast<const uint16_t*>(s + kstep + o * 2);
        if (part == 1) st[u] = s[vstep + o];
      }
      if (part == 0 && i < n) {
        w[u] = w_in[j[u]];
        if (!there) report(a.status, IVIT_ERR_RANGE);
      }
    }
    if (kOrdered) __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kRows + tid / kParts;
      if (i < n && part == 0) w_out[i] = w[u];
      if (dp[u] >= 0) {
        uint8_t* t = a.c.block(dp[u], h);
        const int o = i & (a.c.page - 1);
        *reinterpret_cast<uint4*>(t + o * (D / 2) + 16 * part) = k[u];
        *reinterpret_cast<uint4*>(t + vcode + o * (D / 2) + 16 * part) = v[u];
        if (part == 0) {
          if (D == 128) *reinterpret_cast<uint32_t*>(t + kstep + o * 4) = st[u];
          else *reinterpret_cast<uint16_t*>(t + kstep + o * 2) = (uint16_t)st[u];
        }
        if (part == 1) t[vstep + o] = (uint8_t)st[u];
      }
    }
    if (kOrdered) __syncthreads();
  }
  for (int64_t i = n + (int64_t)blockIdx.x * kThreads + tid; i < a.ldw_out; i += (int64_t)gridDim.x * kThreads) w_out[i] = 0;
  if (h == 0 && blockIdx.x == 0 && tid == 0) a.new_lens[b] = n;
}

int launch_kv4_evict(ivit_ctx* ctx, const ivit_kv4_cache& cache, const ivit_kv4_evict_params& p) {
  const EvictArgs a{to_dev(&cache), p.weights, p.ldw, p.lens, p.table, p.ldtable, p.dst_table, p.ld_dst, p.weights_out, p.ldw_out, p.kept, p.new_lens,
                    (int)p.max_len, (int)p.keep, (int)p.sinks, (int)p.recent, ctx->status_dev};
  int rc;
  {
    LaunchScope ls(ctx, KIND_MOVE, 8.0 * p.seqs * cache.heads * p.max_len);
    const dim3 grid((unsigned)cache.heads, (unsigned)p.seqs);
    if (p.max_len <= 16384) launch_k(kv4_select_kernel<true>, grid, 1024, 0, ctx->stream, a);
    else launch_k(kv4_select_kernel<false>, grid, 1024, 0, ctx->stream, a);
    if ((rc = ls.done())) return rc;
  }
  // in place (of the pages, or of the weights): in order
  const bool ordered = p.dst_table == p.table || p.weights_out == p.weights;
  const int64_t rows = p.keep < p.max_len ? p.keep : p.max_len, per = 4 * 256 / (cache.d / 32);
  const dim3 grid(ordered ? 1u : (unsigned)(rows > per ? (rows + per - 1) / per : 1), (unsigned)cache.heads, (unsigned)p.seqs);
  LaunchScope ls(ctx, KIND_MOVE, 2.0 * p.seqs * cache.heads * rows * (cache.d + cache.d / 32 + 9));
  if (cache.d == 128) ordered ? launch_k(kv4_compact_kernel<128, true>, grid, 512, 0, ctx->stream, a) : launch_k(kv4_compact_kernel<128, false>, grid, 256, 0, ctx->stream, a);
  else ordered ? launch_k(kv4_compact_kernel<64, true>, grid, 512, 0, ctx->stream, a) : launch_k(kv4_compact_kernel<64, false>, grid, 256, 0, ctx->stream, a);
  return ls.done();
}

}  // namespace ivit
