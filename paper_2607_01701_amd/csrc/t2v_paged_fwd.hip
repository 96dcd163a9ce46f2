// Forward kernels of causal attention over a paged cache.
//
// Rows and steps are those of t2v_causal_fwd.hip: packed rows (query, head of the group), 32-key steps of an online softmax on
// keys and values staged through LDS. Here the keys come from pages: a step's keys start at a multiple of 32, pages hold a
// multiple of 16, so every 16 keys lie in one page, whose number is read with scalar loads a step ahead. The work is divided
// by the kernels themselves (t2v_paged.h): each of a fixed number of workgroups takes an even share of all loops.
//
// A page number outside the cache is replaced by a row of NaN, so that it shows in the queries that see it and nothing is read.
#include <algorithm>

#include "t2v_causal_fwd_step.hpp"
#include "t2v_paged_kernels.h"

namespace t2v {

using namespace kern;

namespace {

constexpr int kFewRows = 32, kManyRows = 128;
constexpr float kNan = __builtin_nanf("");
constexpr int kStage = 64;  // keys of an LDS stage of the kernel of 128 rows

typedef __attribute__((address_space(4))) const int32_t const_i32;  // read with scalar loads

struct PagesView {
  const bf16 *k, *v;
  int64_t k_page, k_token, k_head, v_page, v_token, v_head;  // strides in elements
  const_i32* table;
  const_i32* lengths;
  int64_t table_stride;
  int pages, shift, room;
};

// The first piece of a cut tile, for the join.
struct PagedDesc {
  int64_t q0;
  int lq, lk, row0, head, pieces, pad;
};

struct PagedArgs {
  const bf16* q;
  int64_t q_stride;
  const_i32* cu;
  int64_t tokens;
  PagesView c;
  PagedRule rule;
  int nseq, heads, kv_heads, shares;
  float scale;  // times log2 e, positive
  unsigned qkeep, qflip;
  bf16* out;
  float* lse;
  float* partial;
  PagedDesc* desc;
  unsigned long long* trace;
};

__device__ __attribute__((aligned(256))) const uint32_t nan_row[64] = {
#define T2V_NAN8 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u
    T2V_NAN8, T2V_NAN8, T2V_NAN8, T2V_NAN8, T2V_NAN8, T2V_NAN8, T2V_NAN8, T2V_NAN8
#undef T2V_NAN8
};

T2V_DEV int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
T2V_DEV int64_t lane_of(int64_t x, int lane) {
  const uint64_t u = static_cast<uint64_t>(x);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(u), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(u >> 32), lane);
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

T2V_DEV PagedSeq seq_at(const PagedArgs& a, int s) {
  return paged_seq(a.cu[s], a.cu[s + 1], a.c.lengths[s], a.tokens, a.c.room);
}

// This workgroup's share of the line: positions from .. to - 1, the first of which lies in sequence `seq` of key head
// `head`, whose interval begins at `at`.
struct Walk {
  int share, head, seq;
  int64_t at, from, to, length;
};

// Each wave works it out by itself: costs of 64 sequences at a time, their sums over the lanes, and a search.
T2V_DEV Walk find_share(const PagedArgs& a, int lane) {
  const int* cu = (const int*)(a.cu);
  const int* lengths = (const int*)(a.c.lengths);
  Walk w;
  // Workgroup b runs on die b % 8: neighbouring shares, whose tiles read the same keys, on one die.
  const int b = blockIdx.x, n = a.shares, per_die = n / 8;
  w.share = n % 8 == 0 ? (b % 8) * per_die + b / 8 : b;
  auto cost_of = [&](int s) -> int64_t {
    if (s >= a.nseq) return 0;
    return paged_cost(a.rule, paged_tiles(a.rule, paged_seq(cu[s], cu[s + 1], lengths[s], a.tokens, a.c.room)));
  };
  int64_t cost = 0, before = 0, sum = 0;
  auto scan = [&](int s0) {  // cost of sequence s0 + lane, of those before it from s0 on, and of all 64
    cost = cost_of(s0 + lane);
    int64_t x = cost;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up(static_cast<long long>(x), d);
      x += lane >= d ? y : 0;
    }
    before = x - cost;
    sum = lane_of(x, 63);
  };
  int64_t head_cost = 0;
  int s0 = 0;
  for (; s0 < a.nseq; s0 += 64) {
    scan(s0);
    head_cost += sum;
  }
  const int64_t total = head_cost * a.kv_heads;
  w.length = paged_share(a.rule, total, a.shares);
  w.from = w.share * w.length;
  w.to = min(total, w.from + w.length);
  w.head = w.seq = 0;
  w.at = 0;
  if (w.from >= w.to) return w;
  w.head = uniform(static_cast<int>(w.from / head_cost));
  int64_t base = w.head * head_cost;
  s0 = 0;
  if (a.nseq > 64) {
    for (;; s0 += 64) {
      scan(s0);
      if (w.from < base + sum) break;
      base += sum;
    }
  }
  const int64_t rest = w.from - base;
  const unsigned long long hit = __ballot(rest >= before && rest < before + cost);
  const int at = __builtin_ctzll(hit);
  w.seq = s0 + at;
  w.at = base + lane_of(before, at);
  return w;
}

// Runs f(row of the table, sequence, its tiles, head, piece) for every piece of this workgroup's share, and leaves the share's descriptor.
template <typename F>
T2V_DEV void for_pieces(const PagedArgs& a, int lane, F&& f) {
  Walk w = find_share(a, lane);
  bool begun = false;
  while (w.from < w.to) {
    const PagedSeq s = seq_at(a, w.seq);
    const PagedTiles t = paged_tiles(a.rule, s);
    const int64_t cost = paged_cost(a.rule, t);
    if (w.from < w.at + cost) {
      int tile = paged_tile_at(a.rule, t, w.from - w.at);
      for (; tile < t.tiles && w.from < w.to; ++tile) {
        const int64_t at = w.at + paged_before(a.rule, t, tile), end = min(w.to, w.at + paged_before(a.rule, t, tile + 1));
        PagedPiece p;
        if (paged_piece(a.rule, s, t, tile, at, w.from, end, w.length, w.share, &p)) {
          if (p.pieces > 1) {
            begun = true;
            if (threadIdx.x == 0) a.desc[w.share] = {s.q0, s.lq, s.lk, tile * a.rule.tile, w.head, p.pieces, 0};
          }
          f(a.c.table + w.seq * a.c.table_stride, s, t, w.head, p);
        }
        w.from = end;
      }
    }
    w.at += cost;
    if (++w.seq == a.nseq) {
      w.seq = 0;
      ++w.head;
    }
  }
  if (!begun && threadIdx.x == 0) a.desc[w.share].pieces = 0;
}

// Row r of a tile: where it is in [T, H, D] tensors, and the last key that it sees. Rows behind the last repeat it.
T2V_DEV LaneRow row_of(const PagedArgs& a, const PagedSeq& s, const PagedTiles& t, int head, int row) {
  const PackedRow pr = packed_row(min(row, t.rows - 1), a.rule.group);
  return {row < t.rows, pr.query + s.lk - s.lq, head * a.rule.group + pr.head, s.q0 + pr.query};
}

T2V_DEV void load_queries(const PagedArgs& a, const bf16* p, bool ok, int G, bf16x8* qop, int n) {
#pragma unroll
  for (int kk = 0; kk < n; ++kk) {
    u32x4 w = load_raw16(p + kk * 16 + G * 8, ok);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (w[e] & a.qkeep) ^ a.qflip;
    qop[kk] = __builtin_bit_cast(bf16x8, w);
  }
}

// Sixteen keys from key `key` on, a multiple of 16: their page's number.
struct Block16 {
  int key, last;  // the first key that is read, and how many rows follow it (15: all)
};
T2V_DEV Block16 block16(int key, int lk) {
  const int k = min(key, lk - 1);
  return {k, key < lk ? min(lk - 1 - key, 15) : 0};
}
T2V_DEV int page_of(const PagesView& c, const_i32* row, int key, int lk) { return row[block16(key, lk).key >> c.shift]; }

// Address of the block's first key and head (uniform); last: the rows that may be read behind it.
T2V_DEV const char* block_address(const PagesView& c, const bf16* base, int64_t page, int64_t token, int64_t head_offset, int id,
                                  const Block16& b, int* last) {
  const bool ok = static_cast<unsigned>(id) < static_cast<unsigned>(c.pages);
  *last = ok ? b.last : 0;
  const int64_t e = id * page + (b.key & ((1 << c.shift) - 1)) * token + head_offset;
  return ok ? reinterpret_cast<const char*>(base + e) : reinterpret_cast<const char*>(nan_row);
}

// One tensor's pages, seen by one head.
struct HeadPages {
  const bf16* base;
  int64_t page, token, head_offset;
};

// ------------------------------------------------------------------ few rows: single tokens

// Copy of 32 keys by one wave into a swizzled tile; instruction j covers RPI rows of one block of 16.
template <int D>
struct StepDma {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NJ = 32 / RPI;
  int r0;
  uint32_t chunk0;
  T2V_DEV explicit StepDma(int lane) : r0(lane / CPR), chunk0(static_cast<uint32_t>((lane % CPR) ^ swz<D>(lane / CPR))) {}
  T2V_DEV void copy(uint32_t lds, const PagesView& c, const HeadPages& p, const int (&ids)[2], int key0, int lk) const {
    const uint32_t ts = static_cast<uint32_t>(p.token * 2);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Block16 b = block16(key0 + 16 * h, lk);
      int last;
      const char* base = block_address(c, p.base, p.page, p.token, p.head_offset, ids[h], b, &last);
#pragma unroll
      for (int i = 0; i < NJ / 2; ++i) {
        const int j = h * (NJ / 2) + i;
        const uint32_t col = (chunk0 ^ static_cast<uint32_t>(swz<D>(RPI * j))) * 16;
        const int r = min(r0 + RPI * i, last);
#if T2V_CHECKED
        if (!check_row(b.key + r, lk)) {
          dma_lds16_s(nan_row, col, lds + j * 1024);
          continue;
        }
#endif
        dma_lds16_s(base, static_cast<uint32_t>(r) * ts + col, lds + j * 1024);
      }
    }
  }
};

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void paged_few_kernel(const PagedArgs a) {
  constexpr int KK = D / 16, DB = D / 32, R = kFewRows;
  constexpr int kTile = 32 * D;             // elements of a step's K or V
  constexpr int kOps = 2 * StepDma<D>::NJ;  // copies of a step
  __shared__ __attribute__((aligned(1024))) bf16 sKV[4][2][2][kTile];  // [wave][buffer][K, V]
  __shared__ float sM[4][R], sL[4][R];
  const unsigned long long trace_t0 = a.trace != nullptr ? trace_clock() : 0ull;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = uniform(tid >> 6);
  const int G = lane >> 5, l32 = lane & 31;
  const StepDma<D> dma(lane);
  const uint32_t buf = lds_addr(sKV[wave]);
  const uint32_t ko = opnd_lane_off<D>(lane);
  const uint32_t vo0 = rows_lane_off<D>(lane, 0), vo1 = rows_lane_off<D>(lane, 1);
  for_pieces(a, lane, [&](const_i32* table, const PagedSeq& s, const PagedTiles& t, int head, const PagedPiece& p) {
    const int row0 = p.tile * R;
    const LaneRow me = row_of(a, s, t, head, row0 + l32);
    const int lim_lo = __builtin_amdgcn_readlane(me.lim, 0);
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    float m_run = -kInf, l_run = 0.0f;
    const int nsteps = (p.end - p.begin + 31) / 32;
    if (wave < nsteps) {
      const HeadPages kp{a.c.k, a.c.k_page, a.c.k_token, head * a.c.k_head};
      const HeadPages vp{a.c.v, a.c.v_page, a.c.v_token, head * a.c.v_head};
      int ids[2];
      auto find = [&](int n) {
#pragma unroll
        for (int h = 0; h < 2; ++h) ids[h] = page_of(a.c, table, p.begin + n * 32 + 16 * h, s.lk);
      };
      auto fetch = [&](int n, uint32_t b) {
        dma.copy(buf + b * (4 * kTile), a.c, kp, ids, p.begin + n * 32, s.lk);
        dma.copy(buf + b * (4 * kTile) + 2 * kTile, a.c, vp, ids, p.begin + n * 32, s.lk);
      };
      find(wave);
      fetch(wave, 0);
      if (wave + 4 < nsteps) find(wave + 4);
      bf16x8 qop[KK];
      load_queries(a, a.q + me.token * a.q_stride + static_cast<int64_t>(me.head) * D, me.ok, G, qop, KK);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) pin(qop[kk]);  // the loads end here, not between counted copies
      uint32_t b = 0;
      for (int n = wave; n < nsteps; n += 4, b ^= 1) {
        // This wave's reads of the buffer that is filled next have returned: their results are used.
        if (n + 4 < nsteps) {
          fetch(n + 4, b ^ 1);
          if (n + 8 < nsteps) find(n + 8);
          wait_vmcnt<kOps>();
        } else {
          wait_vmcnt0();
        }
        asm volatile("" ::: "memory");
        const uint32_t tile = buf + b * (4 * kTile);
        const uint32_t vb = tile + 2 * kTile;
        const int key0 = p.begin + n * 32;
        if (key0 + 31 <= lim_lo)
          fwd_step<D, false>(tile + ko, vb + vo0, vb + vo1, 0, 0, a.scale, qop, o, m_run, l_run, lane);
        else
          fwd_step<D, true>(tile + ko, vb + vo0, vb + vo1, 0, me.lim - key0, a.scale, qop, o, m_run, l_run, lane);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // before the next copy over what this step read
      }
    }

    // The waves' sums, unnormalised and each with its own reference, in fp32: wave w's in its buffers.
    const float lt = half_sum(l_run);
    float* mine = reinterpret_cast<float*>(sKV[wave]);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = o[db][i * 4 + e];
        *reinterpret_cast<f32x4*>(mine + l32 * D + db * 32 + i * 8 + G * 4) = w;
      }
    if (G == 0) {
      sM[wave][l32] = m_run;
      sL[wave][l32] = lt;
    }
    __syncthreads();
    // A thread takes D / 8 columns of one row.
    constexpr int C = D / 8;
    const int r = tid >> 3, col = (tid & 7) * C;
    const LaneRow row = row_of(a, s, t, head, row0 + r);
    if (row.ok) {
      float m = sM[0][r];
#pragma unroll
      for (int w = 1; w < 4; ++w) m = max_nan(m, sM[w][r]);
      const float ref = m == -kInf ? 0.0f : m;
      float l = 0.0f, x[C];
#pragma unroll
      for (int e = 0; e < C; ++e) x[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(sM[w][r] - ref);
        l = fmaf(f, sL[w][r], l);
        const float* src = reinterpret_cast<const float*>(sKV[w]) + r * D + col;
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = fmaf(f, src[e], x[e]);
      }
      if (p.slot >= 0) {
        float* po = a.partial + static_cast<int64_t>(p.slot) * (R * (D + 2));
#pragma unroll
        for (int e = 0; e < C; e += 4) *reinterpret_cast<f32x4*>(po + r * D + col + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        if (col == 0) {
          po[R * D + 2 * r] = m;
          po[R * D + 2 * r + 1] = l;
        }
      } else {
        const float inv = s.bad ? kNan : row.lim < 0 ? 0.0f : 1.0f / l;
        bf16* op = a.out + (row.token * a.heads + row.head) * D + col;
#pragma unroll
        for (int e = 0; e < C; e += 8) {
          bf16x8 w;
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = static_cast<bf16>(x[e + i] * inv);
          *reinterpret_cast<bf16x8*>(op + e) = w;
        }
        if (col == 0)
          a.lse[static_cast<int64_t>(row.head) * a.tokens + row.token] = s.bad ? kNan : (m + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
    __syncthreads();  // before the next piece's copies over the sums
  });
  if (a.trace != nullptr) trace_end(a.trace, trace_t0, 0, blockIdx.x);
}

// ------------------------------------------------------------------ many rows: chunks and prompts

// Copy of a stage of 64 keys by a workgroup into a swizzled tile: wave w's instruction j covers RPI rows from row RPI (w + NW j) on,
// which lie in one block of 16.
template <int D, int NT>
struct StageDma {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NW = NT / 64, NJ = kStage / RPI / NW;
  static_assert((RPI * NW) % 16 == 0, "a lane's swizzled chunk must not depend on the instruction");
  int wave, r;  // r: this lane's row of its block
  uint32_t col;
  T2V_DEV explicit StageDma(int tid) {
    wave = uniform(tid >> 6);
    const int row = RPI * wave + (tid & 63) / CPR;
    r = row & 15;
    col = static_cast<uint32_t>((((tid & 63) % CPR) ^ swz<D>(row)) * 16);
  }
  T2V_DEV int block(int j) const { return (RPI * (wave + NW * j)) & ~15; }  // its first key
  T2V_DEV void find(int (&ids)[NJ], const PagesView& c, const_i32* table, int key0, int lk) const {
#pragma unroll
    for (int j = 0; j < NJ; ++j) ids[j] = page_of(c, table, key0 + block(j), lk);
  }
  T2V_DEV void copy(bf16* tile, const PagesView& c, const HeadPages& p, const int (&ids)[NJ], int key0, int lk) const {
    const uint32_t ts = static_cast<uint32_t>(p.token * 2);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const Block16 b = block16(key0 + block(j), lk);
      int last;
      const char* base = block_address(c, p.base, p.page, p.token, p.head_offset, ids[j], b, &last);
      const uint32_t lds = lds_addr(tile) + (wave + NW * j) * 1024;
      const int row = min(r, last);
#if T2V_CHECKED
      if (!check_row(b.key + row, lk)) {
        dma_lds16_s(nan_row, col, lds);
        continue;
      }
#endif
      dma_lds16_s(base, static_cast<uint32_t>(row) * ts + col, lds);
    }
  }
};

template <int D>
__global__ __launch_bounds__(256, 2) void paged_many_kernel(const PagedArgs a) {
  constexpr int KK = D / 16, DB = D / 32, NT = 256, R = kManyRows;
  using Dma = StageDma<D, NT>;
  __shared__ __attribute__((aligned(1024))) bf16 sK[2][kStage * D];
  __shared__ __attribute__((aligned(1024))) bf16 sV[2][kStage * D];
  const unsigned long long trace_t0 = a.trace != nullptr ? trace_clock() : 0ull;
  const int tid = threadIdx.x;
  const int wave = uniform(tid >> 6);
  for_pieces(a, tid & 63, [&](const_i32* table, const PagedSeq& s, const PagedTiles& t, int head, const PagedPiece& p) {
    const int lane = lane_again(), G = lane >> 5, l32 = lane & 31;
    const int row0 = p.tile * R + wave * 32;
    const bool wave_active = row0 < t.rows;
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    float m_run = -kInf, l_run = 0.0f;
    const int ntiles = (p.end - p.begin + kStage - 1) / kStage;
    if (ntiles > 0) {
      const LaneRow me = row_of(a, s, t, head, row0 + l32);
      const int lim = me.lim, lim_lo = __builtin_amdgcn_readlane(lim, 0), lim_hi = __builtin_amdgcn_readlane(lim, 31);
      const HeadPages kp{a.c.k, a.c.k_page, a.c.k_token, head * a.c.k_head};
      const HeadPages vp{a.c.v, a.c.v_page, a.c.v_token, head * a.c.v_head};
      const Dma dma(tid);
      int ids[Dma::NJ];
      dma.find(ids, a.c, table, p.begin, s.lk);
      dma.copy(sK[0], a.c, kp, ids, p.begin, s.lk);
      dma.copy(sV[0], a.c, vp, ids, p.begin, s.lk);
      if (ntiles > 1) dma.find(ids, a.c, table, p.begin + kStage, s.lk);
      bf16x8 qop[KK];
      load_queries(a, a.q + me.token * a.q_stride + static_cast<int64_t>(me.head) * D, me.ok, G, qop, KK);
      const uint32_t ko = opnd_lane_off<D>(lane);
      const uint32_t vo0 = rows_lane_off<D>(lane, 0), vo1 = rows_lane_off<D>(lane, 1);
      wait_vmcnt0();
      __syncthreads();
      auto prefetch = [&](int tt) {
        if (tt + 1 < ntiles) {
          const int key0 = p.begin + (tt + 1) * kStage;
          dma.copy(sK[(tt & 1) ^ 1], a.c, kp, ids, key0, s.lk);
          dma.copy(sV[(tt & 1) ^ 1], a.c, vp, ids, key0, s.lk);
          if (tt + 2 < ntiles) dma.find(ids, a.c, table, key0 + kStage, s.lk);
        }
      };
      // Stages that all rows of this wave see whole, then the others: every wave passes ntiles barriers.
      const int nfull = wave_active ? min(max(lim_lo + 1 - p.begin, 0) / kStage, ntiles) : 0;
      int tt = 0;
      for (; tt < nfull; ++tt) {
        const int b = tt & 1;
        prefetch(tt);
        const uint32_t kbase = lds_addr(sK[b]) + ko;
        const uint32_t vb0 = lds_addr(sV[b]) + vo0, vb1 = lds_addr(sV[b]) + vo1;
#pragma unroll
        for (int kb = 0; kb < kStage; kb += 32)
          fwd_step<D, false>(kbase, vb0, vb1, kb, 0, a.scale, qop, o, m_run, l_run, lane);
        wait_vmcnt0();
        __syncthreads();
      }
      for (; tt < ntiles; ++tt) {
        const int b = tt & 1;
        const int key0 = p.begin + tt * kStage;
        prefetch(tt);
        if (wave_active) {
          const uint32_t kbase = lds_addr(sK[b]) + ko;
          const uint32_t vb0 = lds_addr(sV[b]) + vo0, vb1 = lds_addr(sV[b]) + vo1;
#pragma unroll 1
          for (int kb = 0; kb < kStage && key0 + kb <= lim_hi; kb += 32)
            fwd_step<D, true>(kbase, vb0, vb1, kb, lim - key0 - kb, a.scale, qop, o, m_run, l_run, lane);
        }
        wait_vmcnt0();
        __syncthreads();
      }
    }
    if (wave_active) {
      // Worked out again, rather than kept in registers through the loop.
      const int lane = lane_again(), G = lane >> 5, l32 = lane & 31;
      const LaneRow me = row_of(a, s, t, head, row0 + l32);
      const float lt = half_sum(l_run);
      if (p.slot >= 0) {  // one piece: unnormalised sums, reference and sum of each row
        float* po = a.partial + static_cast<int64_t>(p.slot) * (R * (D + 2));
        float* pm = po + R * D;
        const int r = wave * 32 + l32;
        if (me.ok) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              f32x4 w;
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = o[db][i * 4 + e];
              *reinterpret_cast<f32x4*>(po + r * D + db * 32 + i * 8 + G * 4) = w;
            }
          if (G == 0) {
            pm[2 * r] = m_run;
            pm[2 * r + 1] = lt;
          }
        }
      } else {
        // A row that sees no key has no softmax: its output is 0 and its lse -inf.
        const float inv = s.bad ? kNan : me.lim < 0 ? 0.0f : 1.0f / lt;
        bf16* op = a.out + (me.token * a.heads + me.head) * D;
#pragma unroll
        for (int db = 0; db < DB; ++db) store_rows(op + db * 32, o[db], inv, G, me.ok);
        if (me.ok && G == 0)
          a.lse[static_cast<int64_t>(me.head) * a.tokens + me.token] = s.bad ? kNan : (m_run + __builtin_amdgcn_logf(lt)) * kLn2;
      }
    }
  });
  if (a.trace != nullptr) trace_end(a.trace, trace_t0, 0, blockIdx.x);
}

// ------------------------------------------------------------------ join

// What the join needs of one kernel's part.
struct JoinPart {
  const float* partial;
  const PagedDesc* desc;
  int rows, blocks, first;  // rows of a tile; workgroups of a share; this part's first workgroup
};
struct JoinArgs {
  JoinPart part[2];
  int parts, heads, group;
  int64_t tokens;
  bf16* out;
  float* lse;
};

// Joins the pieces of the tile that a share begins: with the largest reference m of a row, out = sum_p 2^(m_p - m) O_p / l,
// l = sum_p 2^(m_p - m) l_p, in piece order. D / 8 lanes hold a row, eight columns each.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const JoinArgs a) {
  constexpr int LPR = D / 8, RPB = kThreads / LPR;
  const bool second = a.parts > 1 && static_cast<int>(blockIdx.x) >= a.part[1].first;
  const JoinPart p = second ? a.part[1] : a.part[0];
  const int b = blockIdx.x - p.first, share = b / p.blocks;
  const PagedDesc it = p.desc[share];
  if (it.pieces == 0) return;
  const int r = (b % p.blocks) * RPB + threadIdx.x / LPR;  // row of the tile
  const int sub = threadIdx.x % LPR, col = sub * 8;
  const int row = it.row0 + r;
  if (row >= it.lq * a.group) return;  // all lanes of a row alike
  const PackedRow pr = packed_row(row, a.group);
  const int64_t slot = static_cast<int64_t>(p.rows) * (D + 2);
  auto piece = [&](int i) { return p.partial + (i == 0 ? 2 * share + 1 : 2 * (share + i)) * slot; };
  const int mo = p.rows * D + 2 * r, xo = r * D + col;
  float m = -kInf;
  for (int i = sub; i < it.pieces; i += LPR) m = max_nan(m, piece(i)[mo]);
#pragma unroll
  for (int off = LPR / 2; off > 0; off >>= 1) m = max_nan(m, __shfl_xor(m, off, LPR));
  const float ref = m == -kInf ? 0.0f : m;
  float l = 0.0f;
  f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
  for (int i0 = 0; i0 < it.pieces; i0 += LPR) {
    const int mine = i0 + sub;
    const bool has = mine < it.pieces;
    const float w_mine = has ? __builtin_amdgcn_exp2f(piece(mine)[mo] - ref) : 0.0f;
    const float l_mine = has ? piece(mine)[mo + 1] : 0.0f;
    const int n = min(LPR, it.pieces - i0);
    for (int i = 0; i < n; ++i) {
      const float w = __shfl(w_mine, i, LPR);
      l = fmaf(w, __shfl(l_mine, i, LPR), l);
      const float* src = piece(i0 + i) + xo;
      const f32x4 u = *reinterpret_cast<const f32x4*>(src);
      const f32x4 v = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = fmaf(w, u[e], x[e]);
        y[e] = fmaf(w, v[e], y[e]);
      }
    }
  }
  const float inv = pr.query + it.lk - it.lq < 0 ? 0.0f : 1.0f / l;
  const int64_t token = it.q0 + pr.query;
  const int head = it.head * a.group + pr.head;
  bf16x8 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = static_cast<bf16>(x[e] * inv);
    w[4 + e] = static_cast<bf16>(y[e] * inv);
  }
  *reinterpret_cast<bf16x8*>(a.out + (token * a.heads + head) * D + col) = w;
  if (col == 0) a.lse[static_cast<int64_t>(head) * a.tokens + token] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ------------------------------------------------------------------ launches

PagedRule rule_of(const PagedCall& c, const PagedPart& p) {
  PagedRule r;
  r.group = c.heads / c.cache.kv_heads;
  r.tile = paged_tile_rows(p.few);
  r.unit = p.few ? 128 : kStage;
  r.least = 128;
  r.fixed = 256;
  r.share = paged_least_share(p.few);
  r.cls = p.cls;
  r.few = kFewRows;
  return r;
}

int64_t desc_bytes(const PagedPart& p) { return (static_cast<int64_t>(p.shares) * sizeof(PagedDesc) + 255) / 256 * 256; }

}  // namespace

int paged_tile_rows(bool few) { return few ? kFewRows : kManyRows; }
int paged_workgroups(bool few, int head_dim, int ncu) { return std::max(1, ncu) * (few ? (head_dim == 64 ? 2 : 1) : 2); }
int paged_least_share(bool few) { return few ? 128 : 128; }
int64_t paged_part_bytes(const PagedPart& p, int head_dim) {
  return desc_bytes(p) + 2 * static_cast<int64_t>(p.shares) * paged_tile_rows(p.few) * (head_dim + 2) * 4;
}

hipError_t launch_paged_fwd(const PagedCall& c, const PagedPart& p, void* ws, hipStream_t s) {
  PagedArgs a{};
  const t2v_pages& g = c.cache;
  a.q = static_cast<const bf16*>(c.q);
  a.q_stride = c.q_stride;
  a.cu = (const_i32*)(c.cu);
  a.tokens = c.tokens;
  a.c.k = static_cast<const bf16*>(g.k);
  a.c.v = static_cast<const bf16*>(g.v);
  a.c.k_page = g.k_strides[0];
  a.c.k_token = g.k_strides[1];
  a.c.k_head = g.k_strides[2];
  a.c.v_page = g.v_strides[0];
  a.c.v_token = g.v_strides[1];
  a.c.v_head = g.v_strides[2];
  a.c.table = (const_i32*)(g.table);
  a.c.lengths = (const_i32*)(g.lengths);
  a.c.table_stride = g.table_stride;
  a.c.pages = static_cast<int>(g.pages);
  a.c.shift = __builtin_ctz(g.page_size);
  a.c.room = g.width * g.page_size;
  a.rule = rule_of(c, p);
  a.nseq = g.nseq;
  a.heads = c.heads;
  a.kv_heads = g.kv_heads;
  a.shares = p.shares;
  // A negative scale turns the sign of Q (so that the largest scaled score is that of the largest product), a scale of 0 clears it.
  a.scale = c.scale == 0.0f ? 1.0f : fabsf(c.scale) * kLog2e;
  a.qkeep = c.scale == 0.0f ? 0u : ~0u;
  a.qflip = c.scale < 0.0f ? 0x80008000u : 0u;
  a.out = static_cast<bf16*>(c.out);
  a.lse = c.lse;
  char* at = static_cast<char*>(ws) + p.at;
  a.desc = reinterpret_cast<PagedDesc*>(at);
  a.partial = reinterpret_cast<float*>(at + desc_bytes(p));
  a.trace = c.trace;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(p.shares), dim3(256), 0, s, a); };
  if (p.few)
    g.head_dim == 128 ? launch(paged_few_kernel<128>) : launch(paged_few_kernel<64>);
  else
    g.head_dim == 128 ? launch(paged_many_kernel<128>) : launch(paged_many_kernel<64>);
  return hipGetLastError();
}

hipError_t launch_paged_join(const PagedCall& c, const PagedPart* parts, int n, void* ws, hipStream_t s) {
  JoinArgs a{};
  const int d = c.cache.head_dim, rows_per_block = kThreads / (d / 8);
  int blocks = 0;
  for (int i = 0; i < n; ++i) {
    char* at = static_cast<char*>(ws) + parts[i].at;
    const int rows = paged_tile_rows(parts[i].few), per = rows / rows_per_block;
    a.part[i] = {reinterpret_cast<const float*>(at + desc_bytes(parts[i])), reinterpret_cast<const PagedDesc*>(at), rows, per, blocks};
    blocks += parts[i].shares * per;
  }
  a.parts = n;
  a.heads = c.heads;
  a.group = c.heads / c.cache.kv_heads;
  a.tokens = c.tokens;
  a.out = static_cast<bf16*>(c.out);
  a.lse = c.lse;
  if (d == 128)
    hipLaunchKernelGGL((paged_join_kernel<128>), dim3(blocks), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((paged_join_kernel<64>), dim3(blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

#if T2V_CHECKED
hipError_t paged_fwd_check_take(unsigned int* rec, unsigned int canary) { return kern::check_take_here(rec, canary); }
#endif
}  // namespace t2v
