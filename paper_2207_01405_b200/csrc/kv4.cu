// A key/value cache held in 4 bits: append to it, eviction from it (sm_100a).  Layout: ivit_kv4_cache in ivit.h.
#include "common.cuh"

namespace ivit {

__device__ __forceinline__ void report(int* status, int code) { *(volatile int*)status = code; }

// One (page, head) block.
struct Block {
  uint8_t* p;
  int d, page;
  __device__ __forceinline__ uint8_t* kcode(int o) const { return p + o * (d / 2); }
  __device__ __forceinline__ uint8_t* kstep(int o) const { return p + page * (d / 2) + o * (d / 32); }
  __device__ __forceinline__ uint8_t* vcode(int o) const { return p + page * (d / 2 + d / 32) + o * (d / 2); }
  __device__ __forceinline__ uint8_t* vstep(int o) const { return p + page * (d + d / 32) + o; }
};

struct Cache {
  uint8_t* data;
  int64_t pages;
  int heads, d, page, page_log;
  __device__ __forceinline__ Block block(int64_t pg, int h) const {
    return Block{data + (pg * heads + h) * ((int64_t)page * (d + d / 32 + 1)), d, page};
  }
};

static Cache to_dev(const ivit_kv4_cache* c) {
  int lg = 0;
  while ((1 << lg) < c->page) ++lg;
  return Cache{c->data, c->pages, (int)c->heads, (int)c->d, (int)c->page, lg};
}

// ---------------------------------------------------------------- append

__device__ __forceinline__ int kv4_code(int x, int step) {
  if (step == 0) return 8;
  return (16 * x + step + 16 * step) / (2 * step);   // + 8 keeps the numerator positive
}

// One warp per (token, head).
__global__ void __launch_bounds__(256) kv4_append_kernel(Cache c, const int8_t* K, int64_t ldk, const int8_t* V, int64_t ldv,
                                                         const int64_t* slots, int64_t tokens, int* status) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t n = tokens * c.heads;
  for (int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; i < n; i += ((int64_t)gridDim.x * blockDim.x) >> 5) {
    const int64_t t = i / c.heads;
    const int h = (int)(i - t * c.heads);
    const int64_t slot = slots[t];
    if (slot < 0) continue;
    if (slot >> c.page_log >= c.pages) {
      if (lane == 0) report(status, IVIT_ERR_RANGE);
      continue;
    }
    const Block b = c.block(slot >> c.page_log, h);
    const int o = (int)(slot & (c.page - 1));
    const int8_t* k = K + t * ldk + h * c.d;
    const int8_t* v = V + t * ldv + h * c.d;
    int vmax = 0;
    for (int ch = lane; ch < c.d; ch += 32) vmax = max(vmax, abs((int)v[ch]));
    vmax = __reduce_max_sync(~0u, vmax);
    const int vs = (8 * vmax + 6) / 7;
    for (int p = lane; p < c.d / 2; p += 32)
      b.vcode(o)[p] = (uint8_t)(kv4_code(v[p], vs) | kv4_code(v[p + c.d / 2], vs) << 4);
    if (lane == 0) *b.vstep(o) = (uint8_t)vs;
    const int G = c.d / 32;
    for (int g = 0; g < G; ++g) {
      const int x = k[32 * g + lane];
      const int ks = (8 * __reduce_max_sync(~0u, abs(x)) + 6) / 7;
      const int lo = kv4_code(x, ks), hi = __shfl_down_sync(~0u, lo, 16);
      if (lane < 16) b.kcode(o)[4 * (G * (lane >> 2) + g) + (lane & 3)] = (uint8_t)(lo | hi << 4);
      if (lane == 0) b.kstep(o)[g] = (uint8_t)ks;
    }
  }
}

int launch_kv4_append(ivit_ctx* ctx, const ivit_kv4_cache* cache, const int8_t* K, int64_t ldk, const int8_t* V, int64_t ldv,
                      const int64_t* slots, int64_t tokens) {
  if (tokens == 0) return IVIT_OK;
  LaunchScope ls(ctx, KIND_MOVE, (double)tokens * cache->heads * 3 * cache->d);
  const int64_t ctas = (tokens * cache->heads + 7) / 8;
  launch_k(kv4_append_kernel, (int)(ctas < 8 * ctx->sm_count ? ctas : 8 * ctx->sm_count), 256, 0, ctx->stream, to_dev(cache), K, ldk, V, ldv,
           slots, tokens, ctx->status_dev);
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

// One CTA per (sequence, head): finds the smallest weight that stays by its bytes from the top, then lists the keys in order.
__global__ void __launch_bounds__(1024) kv4_select_kernel(EvictArgs a) {
  __shared__ unsigned hist[256];
  __shared__ unsigned long long prefix_s;
  __shared__ unsigned need_s;
  __shared__ unsigned sums[32][2];
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
  const int lo = a.sinks, hi = len - a.recent;      // candidates
  unsigned need = (unsigned)(a.keep - a.sinks - a.recent);   // of them
  unsigned long long prefix = 0;
  for (int shift = 56; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += 1024) {
      const unsigned long long k = order_key(w[j]);
      if (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      unsigned n = need;
      int v = 255;
      while (v > 0 && hist[v] < n) n -= hist[v--];
      prefix_s = prefix | (unsigned long long)v << shift;
      need_s = n;
    }
    __syncthreads();
    prefix = prefix_s;
    need = need_s;
  }
  // weights above `prefix` stay, and the first `need` of those equal to it
  int base = 0, ties = 0;
  for (int j0 = 0; j0 < len; j0 += 1024) {
    const int j = j0 + tid;
    bool above = false, tie = false;
    if (j < len) {
      const unsigned long long k = order_key(w[j]);
      above = j < lo || j >= hi || k > prefix;
      tie = !above && k == prefix;
    }
    const unsigned ma = __ballot_sync(~0u, above), mt = __ballot_sync(~0u, tie), below = (1u << lane) - 1;
    if (lane == 0) { sums[warp][0] = __popc(ma); sums[warp][1] = __popc(mt); }
    __syncthreads();
    int nt = ties + __popc(mt & below), na = base + __popc(ma & below), all_a = 0, all_t = 0;
    for (int i = 0; i < 32; ++i) {
      if (i < warp) { na += sums[i][0]; nt += sums[i][1]; }
      all_a += sums[i][0];
      all_t += sums[i][1];
    }
    // (base counts the keys above only; ties in front of this one that stay: min(nt, need))
    const int at = na + min(nt, (int)need);
    if (above || (tie && nt < (int)need)) kept[at] = j;
    base += all_a;
    ties += all_t;
    __syncthreads();
  }
}

// One CTA per (sequence, head) moves the rows in order: rows that are read later lie behind those that are written.
__global__ void __launch_bounds__(256) kv4_compact_kernel(EvictArgs a) {
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  const int h = blockIdx.x, b = blockIdx.y, d = a.c.d;
  const int n = min(evict_len(a, b), a.keep);
  const int64_t bh = (int64_t)b * a.c.heads + h;
  for (int i0 = 0; i0 < n; i0 += 256) {
    const int i = i0 + tid;
    Block s{nullptr, 0, 0}, t{nullptr, 0, 0};
    int so = 0, to = 0;
    int64_t w = 0;
    if (i < n) {
      const int j = a.kept[bh * a.keep + i];
      const int64_t sp = a.table[b * a.ldtable + (j >> a.c.page_log)], dp = a.dst[b * a.ld_dst + (i >> a.c.page_log)];
      w = a.w[bh * a.ldw + j];
      so = j & (a.c.page - 1);
      to = i & (a.c.page - 1);
      if (sp >= 0 && sp < a.c.pages && dp >= 0 && dp < a.c.pages) { s = a.c.block(sp, h); t = a.c.block(dp, h); }
      else report(a.status, IVIT_ERR_RANGE);
    }
    uint4 k[4], v[4];
    unsigned ks = 0, vs = 0;
    if (s.p) {
      for (int q = 0; q < d / 32; ++q) {
        k[q] = reinterpret_cast<const uint4*>(s.kcode(so))[q];
        v[q] = reinterpret_cast<const uint4*>(s.vcode(so))[q];
        ks |= (unsigned)s.kstep(so)[q] << (8 * q);
      }
      vs = *s.vstep(so);
    }
    __syncthreads();
    if (s.p) {
      for (int q = 0; q < d / 32; ++q) {
        reinterpret_cast<uint4*>(t.kcode(to))[q] = k[q];
        reinterpret_cast<uint4*>(t.vcode(to))[q] = v[q];
        t.kstep(to)[q] = (uint8_t)(ks >> (8 * q));
      }
      *t.vstep(to) = (uint8_t)vs;
    }
    if (i < n) a.w_out[bh * a.ldw_out + i] = w;
    __syncthreads();
  }
  for (int64_t i = n + tid; i < a.ldw_out; i += 256) a.w_out[bh * a.ldw_out + i] = 0;
  if (h == 0 && tid == 0) a.new_lens[b] = n;
}

int launch_kv4_evict(ivit_ctx* ctx, const ivit_kv4_cache* cache, const int64_t* weights, int64_t ldw, const int32_t* lens, const int32_t* table,
                     int64_t ldtable, const int32_t* dst_table, int64_t ld_dst, int64_t* weights_out, int64_t ldw_out, int32_t* kept,
                     int32_t* new_lens, int64_t seqs, int64_t max_len, int64_t keep, int64_t sinks, int64_t recent) {
  if (seqs == 0) return IVIT_OK;
  const EvictArgs a{to_dev(cache), weights, ldw, lens, table, ldtable, dst_table, ld_dst, weights_out, ldw_out, kept, new_lens, (int)max_len,
                    (int)keep, (int)sinks, (int)recent, ctx->status_dev};
  const dim3 grid((unsigned)cache->heads, (unsigned)seqs);
  int rc;
  {
    LaunchScope ls(ctx, KIND_MOVE, 8.0 * seqs * cache->heads * max_len);
    launch_k(kv4_select_kernel, grid, 1024, 0, ctx->stream, a);
    if ((rc = ls.done())) return rc;
  }
  LaunchScope ls(ctx, KIND_MOVE, 2.0 * seqs * cache->heads * keep * (cache->d + cache->d / 32 + 9));
  launch_k(kv4_compact_kernel, grid, 256, 0, ctx->stream, a);
  return ls.done();
}

}  // namespace ivit
