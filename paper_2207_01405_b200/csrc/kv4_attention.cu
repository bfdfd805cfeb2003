// Attention of query rows over a key/value cache held in 4 bits (ivit_kv4_attention), sm_100a.
#include "kv4_layout.cuh"
#include "tc_ptx.cuh"

#include <type_traits>

namespace ivit {

struct AttendArgs {
  const uint8_t* data;
  int64_t pages, block_bytes;
  int heads, page, page_log;
  const int8_t* Q; int64_t ldq;
  Kv4Div group;                    // query heads per key/value head
  int64_t tokens;
  const int32_t *q_start, *lens, *table;
  int64_t ldtable;
  int qk_mult, qk_add, qk_sh;      // s = (hi32(16 a qk_mult) + qk_add) >> qk_sh
  unsigned sixteen;                // 16, not known to the compiler: a multiplication where a shift would take the busier unit
  int pv_mult, pv_shift, I0, N, z;
  int8_t* O; int64_t ldo;
  int64_t* weights; int64_t ldw;
  int max_q, max_len, split, blocks, kept, sorted;   // sorted: the number of sequences, which go longest first (0: in their order)
  int* status;
};

// ---------------------------------------------------------------- instructions

// 16 bytes to shared memory where ok, without a branch (which would keep the instructions around it apart).
__device__ __forceinline__ void cp16_if(bool ok, uint32_t dst, const void* src) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst), "l"(src), "r"((int)ok) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_addr(uint32_t a, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
// A value into a peer's shared memory, counted by a barrier of that peer: no fence, no answer to wait for.
__device__ __forceinline__ void send_i32(uint32_t a, int v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.s32 [%0], %1, [%2];" ::"r"(a), "r"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void send_u64(uint32_t a, unsigned long long v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u64 [%0], %1, [%2];" ::"r"(a), "l"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}

// D += A B on 16 x 32 by 32 x 8 bytes; both signed or both unsigned.
template <bool kUnsigned>
__device__ __forceinline__ void mma8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (kUnsigned)
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.u8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Sixteen times the codes of the low (high) halves of four bytes, as signed bytes: code + 8 with its top bit flipped is the code in
// two's complement, and a nibble in the upper half of a byte needs no sign extension.
__device__ __forceinline__ uint32_t low16(uint32_t w, uint32_t sixteen) { return ((w * sixteen) ^ 0x80808080u) & 0xf0f0f0f0u; }
__device__ __forceinline__ uint32_t high16(uint32_t w) { return (w ^ 0x80808080u) & 0xf0f0f0f0u; }

// Four 32-bit values saturated to int8 and packed, x0 in the low byte.
__device__ __forceinline__ uint32_t pack_sat(int x0, int x1, int x2, int x3) {
  uint32_t t, r;
  asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(t) : "r"(x3), "r"(x2), "r"(0));
  asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(x1), "r"(x0), "r"(t));
  return r;
}

// Two 16 x 16 blocks of bytes, transposed on the way from shared memory: lane 4 n + t gets rows 4 t .. 4 t + 3 of columns n (y0) and n + 8
// (y1) of the first, y2 and y3 of the second.  Lane l names row l of the two.
__device__ __forceinline__ void load_transposed(uint32_t addr, uint32_t& y0, uint32_t& y1, uint32_t& y2, uint32_t& y3) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(y0), "=r"(y1), "=r"(y2), "=r"(y3) : "r"(addr) : "memory");
}

// Entry of the exponentials for the score in one byte of w: `sel` holds -4 kKv4Copies in that byte, t = table + copy + 4 kKv4Copies max.
__device__ __forceinline__ unsigned exp_of(uint32_t w, uint32_t sel, uint32_t t) {
  unsigned e;
  asm("{\n\t.reg .u32 a;\n\tdp4a.s32.s32 a, %1, %2, %3;\n\tld.shared.u32 %0, [a];\n\t}" : "=r"(e) : "r"(w), "r"(sel), "r"(t));
  return e;
}

// ---------------------------------------------------------------- the kernel
//
// A cluster of `split` CTAs takes up to 8 RN query rows (of one sequence, all of them readers of one key/value head) and shares the
// keys out in runs of blocks of 32; the warps of a CTA take its blocks in turn.  Two passes, because ShiftExp needs the row's
// maximum before the first weight (its floors do not commute with a change of the maximum, so nothing can be corrected afterwards):
//   scores:  S^T = K Q^T on m16n8k32 products, keys along M, the query rows along N (a decoder has 1 to 16 of them: none is padding of 16).
//            One product of 32 channels is one group of a key, whose step multiplies it in 32 bits; the int8 scores stay in shared memory.
//   values:  O^T = V^T U, channels along M, the weights u (16 bits) as two planes of unsigned bytes.
// A warp brings its codes in with cp.async, kKv4Stages - 1 blocks ahead (the first blocks of V are under way across the exchange of the
// maxima).  K is unpacked in registers, three instructions for eight codes; V's rows are transposed by the loads, and a byte goes into the
// products as it is, or with its lower half cleared: the difference of the two sums is the lower code's.  Maxima, sums and outputs of the
// cluster's CTAs meet in distributed shared memory: one launch, no workspace, and integer sums, so that the order changes nothing.
//
// What bounds it, decoding: 37 sequences of up to 7000 keys, 32 / 8 heads of 128, 139 MB, 33 us (4.2 TB/s, 0.64 of the copy rate): about
// 160 clocks of an SM for 32 keys, in which no unit is busy half of the time (issue 46 % of all cycles, shared memory 38 %, ALU 33 %), and 8000 clocks
// around a CTA's keys (set-up, exponentials, exchange, sums, quotients).  Many query rows (16 a CTA): registers hold the sums, two warps
// for a scheduler do not cover one another's latencies: issue 43 % (5 sequences of up to 300 tokens over up to 2500 keys, 63 us).
template <int D, int RN, int W, bool kWeights>
__global__ void __launch_bounds__(32 * W, RN == 1 && W == 8 ? 2 : 1) kv4_attention_kernel(const AttendArgs a) {
  constexpr int kG = D / 32;               // groups of a key
  constexpr int kLaneWords = D / 32;       // words of a K row that a lane takes
  constexpr int kMu = D / 16;              // tiles of 16 channels
  constexpr int T = 32 * W;                // threads
  constexpr int kRows = 8 * RN, kStage = kKv4Block * (D / 2 + D / 32);
  extern __shared__ __align__(128) uint8_t sm[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n8 = lane >> 2, t4 = lane & 3;
  const int rank = blockIdx.x % a.split, tile = blockIdx.x / a.split, h = blockIdx.y;
  int b = blockIdx.z;
  const Kv4Smem at = kv4_smem(D, kRows, a.kept, a.page, a.blocks, a.split, W);
  const uint8_t** const pages = reinterpret_cast<const uint8_t**>(sm + at.pages);   // this head's block of each page of the run
  int* const small = reinterpret_cast<int*>(sm + at.small);
  int* const lim = small;                                                            // [16] keys that a row sees
  int* const top = small + 16;                                                       // [16] maxima of the rows
  int* const warp_top = small + 32;                                                  // [16][16]
  int* const cta_u = small + 288;                                                    // [2][16] sums of the weights' planes
  unsigned long long* const row_den = reinterpret_cast<unsigned long long*>(small + 320);   // [16]
  unsigned long long* const row_u = row_den + 16;                                    // [16]
  unsigned long long* const row_recip = row_u + 16;                                  // [16]
  unsigned long long* const row_out = row_recip + 16;                                // [16] where a row of O starts
  unsigned long long* const warp_den = row_out + 16;                                 // [16][16]
  const uint32_t bar0 = smem_u32(warp_den + 256), bar1 = bar0 + 8;                   // what peers send: maxima; sums
  static_assert(4 * 320 + 8 * (4 * 16 + 256 + 2) <= kKv4Small, "room for the rows' numbers");
  int* const sums = reinterpret_cast<int*>(sm + at.sums);                            // [plane][row][channel]
  // what the CTAs of the cluster send: [rank][row] maxima, [denominator, weights][rank][row], [rank][this CTA's share of the sums]
  int* const top_in = reinterpret_cast<int*>(sm + at.peers);
  unsigned long long* const row_in = reinterpret_cast<unsigned long long*>(sm + at.peers + 4 * 16 * kRows);
  long long* const part_in = reinterpret_cast<long long*>(row_in + 2 * 16 * kRows);
  const int score_ld = kv4_score_ld(a.blocks);
  int8_t* const score = reinterpret_cast<int8_t*>(sm + at.score);
  constexpr int kLd = D + 4;
  // what needs nothing that a kernel in front may still be writing
  for (int i = tid; i < 2 * kRows * kLd / 4; i += T) reinterpret_cast<int4*>(sums)[i] = make_int4(0, 0, 0, 0);
  if (tid < 32) cta_u[tid] = 0;
  if (a.split > 1) {
    if (tid == 0) {
      mbar_init(bar0, 1);
      mbar_init(bar1, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_arrive();
  }
  if (tid < 256) {  // the exponentials, shifted so that a weight's 16 bits are the upper half of its product with a step
    const unsigned e = shiftexp(-tid, a.I0, a.N) << (16 - a.z);
    uint4* dst = reinterpret_cast<uint4*>(sm + at.table) + tid * (kKv4Copies / 4);
    static_assert(kKv4Copies % 4 == 0, "whole vectors");
#pragma unroll
    for (int i = 0; i < kKv4Copies / 4; ++i) dst[i] = make_uint4(e, e, e, e);
  }
  const int row0 = tile * kRows;
  int q_at[RN], q_head[RN];                            // query token and head (of the group's) of the lane's rows
#pragma unroll
  for (int j = 0; j < RN; ++j) {
    q_at[j] = a.group.div(row0 + 8 * j + n8);
    q_head[j] = row0 + 8 * j + n8 - q_at[j] * (int)a.group.d;
  }
  pdl_wait();
  pdl_trigger();
  if (a.sorted) {
    // The z-th longest sequence (of equal ones the one in front): a long one that starts behind the others would end long after them.
    int* const order = reinterpret_cast<int*>(score);
    if (tid < a.sorted) order[tid] = a.lens[tid];
    __syncthreads();
    if (tid < a.sorted) {
      const int mine = order[tid];
      int before = 0;
      for (int i = 0; i < a.sorted; ++i) before += order[i] > mine || (order[i] == mine && i < tid);
      if (before == b) top[0] = tid;
    }
    __syncthreads();
    b = top[0];
    __syncthreads();
  }
  // (not split: the first pages are known without the lengths, and fetched beside them)
  const int early = a.split == 1 && (tid << a.page_log) < a.max_len ? a.table[b * a.ldtable + tid] : 0;
  const Kv4Seq seq = kv4_sequence(a.q_start[b], a.q_start[b + 1], a.lens[b], a.tokens, a.max_q, a.max_len);
  if (seq.bad && tid == 0) *(volatile int*)a.status = IVIT_ERR_RANGE;
  const int nrows = min(kRows, seq.n * (int)a.group.d - row0);
  if (nrows <= 0) {                        // (the whole cluster)
    if (a.split > 1) cluster_wait();
    return;
  }
  // keys that some row of the tile sees, and this CTA's run of them
  const int seen_all = kv4_seen(seq, a.group.div(row0 + nrows - 1)), seen_min = kv4_seen(seq, a.group.div(row0));
  const int blks = (seen_all + kKv4Block - 1) / kKv4Block;
  // A sequence takes as many of the cluster's CTAs as leave each no more than the launch was sized for: short ones among long ones pay for
  // no exchange, and their CTAs make room.
  const int split = max(1, min(a.split, (blks + a.blocks - 1) / a.blocks));
  if (rank >= split) {
    cluster_wait();
    return;
  }
  const int run = (blks + split - 1) / split;
  // sums that a CTA finishes, in the order [row][channel], and those that are left for this one
  const int own = (kRows * D + split - 1) / split, mine_n = max(0, min(own, kRows * D - rank * own));
  if (split > 1 && tid == 0) {
    expect_bytes(bar0, 4 * split * kRows);
    expect_bytes(bar1, 16 * split * kRows + 8 * split * mine_n);
  }
  const int blk0 = rank * run, nblk = max(0, min(run, blks - blk0));
  const int page0 = blk0 * kKv4Block >> a.page_log;
  bool bad = false;
  for (int i = tid; i < (nblk > 0 ? ((blk0 + nblk) * kKv4Block - 1 >> a.page_log) - page0 + 1 : 0); i += T) {
    const int pg = a.split == 1 && i < T ? early : a.table[b * a.ldtable + page0 + i];
    const bool there = pg >= 0 && pg < a.pages;
    if (!there) {
      bad = true;
      *(volatile int*)a.status = IVIT_ERR_RANGE;
    }
    pages[i] = there ? a.data + ((int64_t)pg * a.heads + h) * a.block_bytes : nullptr;
  }
  if (t4 == 0 && warp == 0)
#pragma unroll
    for (int j = 0; j < RN; ++j) {
      lim[8 * j + n8] = 8 * j + n8 < nrows ? kv4_seen(seq, q_at[j]) : 0;
      row_out[8 * j + n8] = (unsigned long long)((seq.q0 + q_at[j]) * a.ldo + (int64_t)(h * (int)a.group.d + q_head[j]) * D);
    }
  // B operand of the scores: the lane's query row of each tile of eight, bytes 32 g + 4 t.. and 32 g + 16 + 4 t..
  uint32_t q[RN][kG][2];
#pragma unroll
  for (int j = 0; j < RN; ++j) {
    const bool there = 8 * j + n8 < nrows;
    const int8_t* src = a.Q + (there ? (seq.q0 + q_at[j]) * a.ldq + (int64_t)(h * (int)a.group.d + q_head[j]) * D : 0) + 4 * t4;
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      q[j][g][0] = there ? *reinterpret_cast<const uint32_t*>(src + 32 * g) : 0;
      q[j][g][1] = there ? *reinterpret_cast<const uint32_t*>(src + 32 * g + 16) : 0;
    }
  }
  const bool holes = __syncthreads_or(bad) != 0;   // a page of the run points nowhere: its keys are not seen

  uint8_t* const ring = sm + at.ring + warp * (kKv4Stages * kStage);
  // A block's codes lie in the ring as rows of 16-byte chunks, at a place of their own for each (row, chunk) that keeps three kinds of
  // access off the same banks: eight rows one behind the other (V, transposed), every fourth row (K), and the rows as they come in.
  auto place = [](int row, int chunk) {
    return D == 128 ? 64 * (row ^ (row >> 2 & 1)) + 16 * (chunk ^ (row >> 1 & 3)) : 32 * (row ^ (row >> 2 & 3)) + 16 * (chunk ^ (row >> 2 & 1));
  };
  const uint32_t ring32 = smem_u32(ring), put = ring32 + place(lane / (D / 32), lane % (D / 32)), put_step = ring32 + kKv4Block * (D / 2) + 16 * lane;
  const int in_page = a.page / kKv4Block - 1, per_page = a.page_log - 5;
  // page and place in it of the run's block lb: pages[(lb + first) >> per_page], (lb + first) & in_page
  const int first = blk0 & in_page;
  const int kcode = kv4_kcode(D, a.page, 0), kstep = kv4_kstep(D, a.page, 0), vcode = kv4_vcode(D, a.page, 0), vstep = kv4_vstep(D, a.page, 0);
  auto page_of = [&](int lb) { return lb < nblk ? pages[(lb + first) >> per_page] : nullptr; };
  auto request = [&](int lb, const uint8_t* src, uint32_t stage, int code, int step, int step_bytes) {
    const int o = (lb + first) & in_page;
    const uint8_t* from = src + (code + o * (kKv4Block * D / 2) + 16 * lane);
#pragma unroll
    for (int i = 0; i < D / 64 * 2; ++i) cp16_if(src != nullptr, put + stage + 512 * i, from + 512 * i);
    cp16_if(src != nullptr && lane < step_bytes / 16, put_step + stage, src + (step + o * step_bytes + 16 * lane));
    cp_commit();
  };
  auto request_k = [&](int lb, const uint8_t* src, uint32_t stage) { request(lb, src, stage, kcode, kstep, kKv4Block * kG); };
  auto request_v = [&](int lb, const uint8_t* src, uint32_t stage) { request(lb, src, stage, vcode, vstep, kKv4Block); };

  // where the lane's parts of K rows 4 n8 + i lie, and its row of V, chunk by chunk
  int k_at[4], v_at[D / 32];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = D == 128 ? place(4 * n8 + i, t4) : place(4 * n8 + i, t4 >> 1) + 8 * (t4 & 1);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) v_at[c] = place(lane, c);

  // ---- scores
  for (int s = 0; s < kKv4Stages - 1; ++s) request_k(warp + W * s, page_of(warp + W * s), s * kStage);
  int best[RN][2];
#pragma unroll
  for (int j = 0; j < RN; ++j) best[j][0] = best[j][1] = -128;
  constexpr int ahead = W * (kKv4Stages - 1);
  constexpr uint32_t last = (kKv4Stages - 1) * kStage;
  uint32_t stage = 0, behind = last;                        // the block at hand; where the one requested now goes
  const uint8_t* next = page_of(warp + ahead);             // (looked up a turn before it is needed)
  for (int lb = warp; lb < nblk; lb += W) {
    cp_wait<kKv4Stages - 2>();
    __syncwarp();
    const uint8_t* buf = ring + stage;
    // what the turn reads, then the request, then the arithmetic: the first is on its way while the second is issued
    uint32_t w[4][kLaneWords];      // the lane's words of K rows 4 n8 + i
    int step[4][kG];                // their steps, byte by byte: the unit of shared memory has time for that, the one that would take words apart has not
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (D == 128) {
        const uint4 v = *reinterpret_cast<const uint4*>(buf + k_at[i]);
        w[i][0] = v.x; w[i][1] = v.y; w[i][kLaneWords - 2] = v.z; w[i][kLaneWords - 1] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(buf + k_at[i]);
        w[i][0] = v.x; w[i][1] = v.y;
      }
#pragma unroll
      for (int g = 0; g < kG; ++g) step[i][g] = buf[kKv4Block * (D / 2) + (4 * n8 + i) * kG + g];
    }
    request_k(lb + ahead, next, behind);
    next = page_of(lb + ahead + W);
    behind = stage;
    stage = stage == last ? 0 : stage + kStage;
    const int key0 = (blk0 + lb) * kKv4Block;
    if (holes && !page_of(lb)) continue;
    int acc[RN][2][4];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int j = 0; j < RN; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][m][i] = 0;
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const uint32_t a0 = low16(w[2 * m][g], a.sixteen), a1 = low16(w[2 * m + 1][g], a.sixteen), a2 = high16(w[2 * m][g]), a3 = high16(w[2 * m + 1][g]);
#pragma unroll
        for (int j = 0; j < RN; ++j) {
          int c[4] = {0, 0, 0, 0};
          mma8<false>(c, a0, a1, a2, a3, q[j][g][0], q[j][g][1]);
          acc[j][m][0] += c[0] * step[2 * m][g];
          acc[j][m][1] += c[1] * step[2 * m][g];
          acc[j][m][2] += c[2] * step[2 * m + 1][g];
          acc[j][m][3] += c[3] * step[2 * m + 1][g];
        }
      }
    }
    auto keep = [&](auto whole) {
#pragma unroll
      for (int j = 0; j < RN; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          int v[4];   // keys 4 n8 .. 4 n8 + 3 of row 2 t4 + e
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = mad_hi(acc[j][i >> 1][2 * (i & 1) + e], a.qk_mult, a.qk_add) >> a.qk_sh;
          const int row = 8 * j + 2 * t4 + e;
          if (!decltype(whole)::value) {   // what the row does not see: a score that is no larger than any, and whose weight is left out below
            const int left = lim[row] - key0 - 4 * n8;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = i < left ? v[i] : -128;
          }
          best[j][e] = max(max(best[j][e], max(v[0], v[1])), max(v[2], v[3]));
          if (row < a.kept) *reinterpret_cast<uint32_t*>(score + row * score_ld + lb * kKv4Block + 4 * n8) = pack_sat(v[0], v[1], v[2], v[3]);
        }
    };
    if (key0 + kKv4Block <= seen_min) keep(std::true_type{});
    else keep(std::false_type{});
  }
  cp_wait<0>();
  __syncwarp();
  for (int s = 0; s < kKv4Stages - 1; ++s) request_v(warp + W * s, page_of(warp + W * s), s * kStage);
  next = page_of(warp + ahead);
#pragma unroll
  for (int j = 0; j < RN; ++j)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      int v = min(best[j][e], 127);
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
      if (lane < 4) warp_top[warp * 16 + 8 * j + 2 * lane + e] = v;
    }
  __syncthreads();
  // sixteen lanes for a row: over the warps of the CTA, then over the CTAs of the cluster
  const int pr = tid >> 4, pk = tid & 15;
  if (a.split > 1) cluster_wait();         // (the peers' barriers are set up)
  if (pr < kRows) {
    int v = pk < W ? warp_top[pk * 16 + pr] : -128;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
    if (split == 1) {
      if (pk == 0) top[pr] = v;
    } else if (pk < split) {
      send_i32(peer_addr(smem_u32(top_in + rank * kRows + pr), pk), v, peer_addr(bar0, pk));
    }
    if (split > 1) {
      const bool arrived = mbar_wait(bar0, 0, a.status);
      v = pk < split ? kv4_peer_top(arrived, top_in[pk * kRows + pr]) : -128;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) v = max(v, __shfl_xor_sync(~0u, v, o));
      if (pk == 0) top[pr] = v;
    }
  }
  __syncthreads();

  // ---- values
  int lo[RN][kMu][4], hi[RN][kMu][4];
  unsigned long long den[RN];
  unsigned ul[RN], uh[RN];                 // sums of the weights' planes
  uint32_t tab[RN];
  const int8_t* mine[RN];                  // the lane's row of scores (rows that no sequence has: the last one that some can have)
  const uint32_t tab0 = smem_u32(sm + at.table) + 4 * (lane & (kKv4Copies - 1));
#pragma unroll
  for (int j = 0; j < RN; ++j) {
    den[j] = ul[j] = uh[j] = 0;
    const int row = min(8 * j + n8, a.kept - 1);
    mine[j] = score + row * score_ld + 4 * t4;
    tab[j] = tab0 + (uint32_t)(4 * kKv4Copies * top[row]);
#pragma unroll
    for (int m = 0; m < kMu; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) lo[j][m][i] = hi[j][m][i] = 0;
  }
  constexpr uint32_t kSel = (uint32_t)(-4 * kKv4Copies) & 255u;
  stage = 0, behind = last;
  for (int lb = warp; lb < nblk; lb += W) {
    cp_wait<kKv4Stages - 2>();
    __syncwarp();
    const uint8_t* buf = ring + stage;
    uint32_t sc[RN][2], vs[2][4], y[D / 32][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int j = 0; j < RN; ++j) sc[j][k] = *reinterpret_cast<const uint32_t*>(mine[j] + lb * kKv4Block + 16 * k);   // keys 4 t4 .., 16 + 4 t4 ..
#pragma unroll
      for (int i = 0; i < 4; ++i) vs[k][i] = buf[kKv4Block * (D / 2) + 16 * k + 4 * t4 + i];                           // their steps
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c) load_transposed(smem_u32(buf) + v_at[c], y[c][0], y[c][1], y[c][2], y[c][3]);
    request_v(lb + ahead, next, behind);
    next = page_of(lb + ahead + W);
    behind = stage;
    stage = stage == last ? 0 : stage + kStage;
    const int key0 = (blk0 + lb) * kKv4Block;
    if (holes && !page_of(lb)) continue;
    uint32_t bl[RN][2], bh[RN][2];   // B operands: word 0 holds keys 4 t4 .., word 1 keys 16 + 4 t4 ..
    auto weigh = [&](auto whole) {
#pragma unroll
      for (int j = 0; j < RN; ++j) {
        unsigned sum = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          unsigned e[4], p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] = exp_of(sc[j][k], kSel << (8 * i), tab[j]);
          if (!decltype(whole)::value) {
            const int left = lim[min(8 * j + n8, a.kept - 1)] - key0 - 4 * t4 - 16 * k;
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = i < left ? e[i] : 0;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sum += e[i];
            p[i] = e[i] * vs[k][i] + 0x8000u;
          }
          const uint32_t p01 = __byte_perm(p[0], p[1], 0x7362), p23 = __byte_perm(p[2], p[3], 0x7362);
          bl[j][k] = __byte_perm(p01, p23, 0x5410);
          bh[j][k] = __byte_perm(p01, p23, 0x7632);
          ul[j] = __dp4a(bl[j][k], 0x01010101u, ul[j]);
          uh[j] = __dp4a(bh[j][k], 0x01010101u, uh[j]);
        }
        den[j] += sum;
      }
    };
    if (key0 + kKv4Block <= seen_min) weigh(std::true_type{});
    else weigh(std::false_type{});
    // 16 bytes of V's rows at a time: byte p holds channels p and p + D/2, so that a tile of 16 bytes is 8 + 8 rows of each of two tiles
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      // 16 (code + 8) of the upper halves' channels; whole bytes, from whose sums those of the upper halves are taken away in the end, for the lower
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t mask = half ? 0xf0f0f0f0u : ~0u;
#pragma unroll
        for (int j = 0; j < RN; ++j) {
          mma8<true>(lo[j][2 * c + half], y[c][0] & mask, y[c][1] & mask, y[c][2] & mask, y[c][3] & mask, bl[j][0], bl[j][1]);
          mma8<true>(hi[j][2 * c + half], y[c][0] & mask, y[c][1] & mask, y[c][2] & mask, y[c][3] & mask, bh[j][0], bh[j][1]);
        }
      }
    }
  }
  cp_wait<0>();

  // ---- the CTA's sums, in shared memory: the warps add theirs (32 different banks at a time)
#pragma unroll
  for (int j = 0; j < RN; ++j) {
    unsigned long long v = den[j];
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      v += __shfl_xor_sync(~0u, v, o);
      ul[j] += __shfl_xor_sync(~0u, ul[j], o);
      uh[j] += __shfl_xor_sync(~0u, uh[j], o);
    }
    if (t4 == 0) {
      warp_den[warp * 16 + 8 * j + n8] = v;
      atomicAdd(cta_u + 8 * j + n8, (int)ul[j]);
      atomicAdd(cta_u + 16 + 8 * j + n8, (int)uh[j]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      int* dst = sums + (8 * j + 2 * t4 + (e & 1)) * kLd + 8 * (e >> 1) + n8;
#pragma unroll
      for (int m = 0; m < kMu; ++m) {
        atomicAdd(dst + (m & 1) * (D / 2) + 16 * (m >> 1), lo[j][m][e]);
        atomicAdd(dst + kRows * kLd + (m & 1) * (D / 2) + 16 * (m >> 1), hi[j][m][e]);
      }
    }
  }
  __syncthreads();
  // ---- the rows' sums and the cluster's
  constexpr int kTurns = kRows * D / T;
  long long part[kTurns];
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int item = tid + T * i;
    const int* src = sums + item / D * kLd + item % D;
    part[i] = src[0] + 256ll * src[kRows * kLd];
    if (item % D < D / 2) part[i] -= src[D / 2] + 256ll * src[kRows * kLd + D / 2];
    if (split > 1) {
      const int to = item / own;
      send_u64(peer_addr(smem_u32(part_in + rank * own + (item - to * own)), to), (unsigned long long)part[i], peer_addr(bar1, to));
    }
  }
  if (pr < kRows) {
    unsigned long long row_d = pk < W ? warp_den[pk * 16 + pr] : 0;   // denominator and sum of the weights, of this CTA
    unsigned long long row_s = (unsigned)cta_u[pr] + 256ull * (unsigned)cta_u[16 + pr];
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) row_d += __shfl_xor_sync(~0u, row_d, o);
    if (split > 1) {
      if (pk < split) {
        send_u64(peer_addr(smem_u32(row_in + rank * kRows + pr), pk), row_d, peer_addr(bar1, pk));
        send_u64(peer_addr(smem_u32(row_in + (16 + rank) * kRows + pr), pk), row_s, peer_addr(bar1, pk));
      }
      mbar_wait(bar1, 0, a.status);
      row_d = pk < split ? row_in[pk * kRows + pr] : 0;
      row_s = pk < split ? row_in[(16 + pk) * kRows + pr] : 0;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        row_d += __shfl_xor_sync(~0u, row_d, o);
        row_s += __shfl_xor_sync(~0u, row_s, o);
      }
    }
    if (pk == 0) {
      row_d >>= 16 - a.z;
      row_den[pr] = row_d;
      row_u[pr] = row_s;
      row_recip[pr] = recip_of(row_d);
    }
  }
  if (split > 1) {
    mbar_wait(bar1, 0, a.status);
    cluster_arrive();                      // (waited for at the end: no CTA leaves while a peer may still send to it, not even when a wait gave up)
#pragma unroll
    for (int i = 0; i < kTurns; ++i)
      if (tid + T * i < mine_n) {
        long long v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = k < split ? part_in[k * own + tid + T * i] : 0;
        part[i] = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) part[i] += v[k];
      }
  }
  __syncthreads();

  // ---- outputs
#pragma unroll
  for (int i = 0; i < kTurns; ++i) {
    const int item = min(rank * own + tid + T * i, kRows * D - 1), row = item / D;
    const int ch = item % D;
    const unsigned long long den_row = row_den[row];
    // (codes came in as code + 8, the upper half's sixteenfold; a row that sees nothing: every number is zero)
    const long long num = (part[i] >> (ch < D / 2 ? 0 : 4)) - 8 * (long long)row_u[row];
    const int t = small_quotient(num * (1ll << (a.z + 5)), den_row, row_recip[row]);
    if (tid + T * i < mine_n && row < nrows) a.O[row_out[row] + ch] = (int8_t)sat8(rq(t, a.pv_mult, a.pv_shift));
  }

  // ---- accumulated weights: floor(e 2^24 / den) of every difference of scores, row by row, then the sum over the rows of each key
  if (kWeights) {
    unsigned* share = reinterpret_cast<unsigned*>(sm + at.ring);
    for (int i = tid; i < nrows * 256; i += T) {
      const unsigned long long den_row = row_den[i >> 8];
      const unsigned e = *reinterpret_cast<const unsigned*>(sm + at.table + (i & 255) * (4 * kKv4Copies)) >> (16 - a.z);
      share[i] = den_row ? (unsigned)small_quotient((long long)e << 24, den_row, row_recip[i >> 8]) : 0;
    }
    __syncthreads();
    unsigned long long* w = reinterpret_cast<unsigned long long*>(a.weights) + ((int64_t)b * a.heads + h) * a.ldw;
    for (int i = tid; i < nblk * 8; i += T) {
      const int key0 = (blk0 + (i >> 3)) * kKv4Block, n = i & 7;
      if (holes && !page_of(i >> 3)) continue;
      unsigned long long v[4] = {0, 0, 0, 0};
      for (int row = 0; row < nrows; ++row) {
        const uint32_t s = *reinterpret_cast<const uint32_t*>(score + row * score_ld + 4 * i);
        const int left = lim[row] - key0 - 4 * n, base = top[row];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < left) v[k] += share[row * 256 + base - (int)(int8_t)(s >> (8 * k))];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (v[k]) atomicAdd(w + key0 + 4 * n + k, v[k]);
    }
  }
  if (split > 1) cluster_wait();
}

// f(kernel, head dimension, query rows, warps, weights) for each of the kernels.
template <class F>
static int each_kernel(F f) {
  int rc = IVIT_OK;
  auto both = [&](auto d, auto rn, auto w) {
    constexpr int D = decltype(d)::value, RN = decltype(rn)::value, W = decltype(w)::value;
    if (rc == IVIT_OK) rc = f(kv4_attention_kernel<D, RN, W, false>, D, 8 * RN, W, false);
    if (rc == IVIT_OK) rc = f(kv4_attention_kernel<D, RN, W, true>, D, 8 * RN, W, true);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, 8> w8;
  const std::integral_constant<int, 16> w16;
  const std::integral_constant<int, 64> d64;
  const std::integral_constant<int, 128> d128;
  both(d64, one, w8); both(d64, one, w16); both(d64, two, w8);
  both(d128, one, w8); both(d128, one, w16); both(d128, two, w8);
  return rc;
}

int kv4_prepare_device(ivit_ctx* ctx) {
  const int rc = each_kernel([](auto k, int, int, int, bool) {
    if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kKv4SmemMax) != cudaSuccess ||
        cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return (int)IVIT_ERR_CUDA;
    return (int)IVIT_OK;
  });
  if (rc) return rc;
  // how many clusters of each size run at once, an SM for each CTA
  for (int c = 1; c <= 16; ++c) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = (unsigned)(c * ctx->sm_count);
    cfg.blockDim = 512;
    cfg.dynamicSmemBytes = kKv4SmemMax;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&ctx->cluster_room[c], kv4_attention_kernel<128, 1, 16, false>, &cfg) != cudaSuccess) {
      cudaGetLastError();
      ctx->cluster_room[c] = c == 1 ? ctx->sm_count : 0;
    }
  }
  return IVIT_OK;
}

int launch_kv4_attention(ivit_ctx* ctx, const ivit_kv4_cache& cache, const ivit_kv4_attention_params& c) {
  const int d = (int)cache.d, page = (int)cache.page;
  const int64_t group = c.q_heads / cache.heads;
  const Kv4Plan p = kv4_plan(d, page, group, cache.heads, c.seqs, c.max_q, c.max_len, ctx->sm_count, ctx->cluster_room);
  if (p.smem > kKv4SmemMax || (int64_t)p.tiles * p.split > 0x7fffffffll) return IVIT_ERR_UNSUPPORTED;
  AttendArgs a{};
  a.data = cache.data; a.pages = cache.pages; a.block_bytes = kv4_block_bytes(d, page);
  a.heads = (int)cache.heads; a.page = page;
  while ((1 << a.page_log) < page) ++a.page_log;
  a.Q = c.Q; a.ldq = c.ldq; a.group = kv4_div((unsigned)group); a.tokens = c.tokens;
  a.q_start = c.q_start; a.lens = c.lens; a.table = c.table; a.ldtable = c.ldtable;
  // rq(x; m, s) = rq(16 x; m, s + 4), whose shift is beyond 32: the rounding constant is a whole number in the product's upper word.  Beyond a
  // shift of 59 every value rounds to zero (|16 x| < 2^30, m < 2^31).
  const int s16 = c.qk_scale.shift + 4;
  a.qk_mult = s16 <= 63 ? c.qk_scale.mult : 0;
  a.qk_add = s16 <= 63 ? 1 << (s16 - 33) : 0;
  a.qk_sh = s16 <= 63 ? s16 - 32 : 0;
  a.sixteen = 16;
  a.pv_mult = c.pv_scale.mult; a.pv_shift = c.pv_scale.shift; a.I0 = c.smax.I0; a.N = c.smax.N;
  const int64_t top = (int64_t)c.smax.I0 << c.smax.N;
  while (top >> (a.z + 8)) ++a.z;
  a.O = c.O; a.ldo = c.ldo; a.weights = c.weights; a.ldw = c.ldw;
  a.max_q = (int)c.max_q; a.max_len = (int)c.max_len; a.split = p.split; a.blocks = p.blocks; a.kept = p.kept;
  // Few waves of long CTAs go longest first, 8 heads, us / in their order: sequences of up to 7000 keys 20 of them 24.1 / 26.0, 25 24.5 / 34.1, 37 32.5 / 40.0,
  // 55 49 / 55; of up to 3000 37 20.8 / 24.0; of up to 12 000 100 130 / 134.  It takes 0.2 us to find a CTA's sequence (the lengths wait where the scores will be).
  const int64_t ctas = cache.heads * c.seqs;
  a.sorted = p.warps == 16 && p.split == 1 && p.tiles == 1 && ctas > ctx->sm_count && c.seqs <= 128 ? (int)c.seqs : 0;
  a.status = ctx->status_dev;
  LaunchScope ls(ctx, KIND_ATTENTION, 4.0 * c.seqs * c.q_heads * c.max_q * c.max_len * d);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.tiles * p.split), (unsigned)cache.heads, (unsigned)c.seqs);
  cfg.blockDim = 32 * p.warps;
  cfg.dynamicSmemBytes = (size_t)p.smem;
  cfg.stream = ctx->stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  each_kernel([&](auto k, int kd, int rows, int warps, bool w) {
    if (kd == d && rows == p.rows && warps == p.warps && w == (c.weights != nullptr)) cudaLaunchKernelEx(&cfg, k, a);
    return (int)IVIT_OK;
  });
  return ls.done();
}

}  // namespace ivit
