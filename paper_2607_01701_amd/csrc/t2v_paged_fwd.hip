// Forward kernels of causal attention over a paged cache.
//
// Rows and steps are those of t2v_causal_fwd.hip: packed rows (query, head of the group), 32-key steps of an online softmax on
// keys and values staged through LDS. Here the keys come from pages: a step's keys start at a multiple of 32, pages hold a
// multiple of 16, so every 16 keys lie in one page, whose number is read with scalar loads a step ahead. The work is divided
// by the kernels themselves (t2v_paged.h): each of a fixed number of workgroups takes an even share of all loops.
//
// A page number outside the cache is replaced by a row of NaN, so that it shows in the queries that see it and nothing is read.
//
// What bounds it. Few rows (single tokens): memory. 32 tokens over 31 to 20,280 keys, 40 heads over 8 of 128, 813 MB: 141 us, 5.75 TB/s; a
// token over 100,000 keys, 24 heads over 8: 70 us; both and the join's 5. Copies to LDS reach 6.0 TB/s, and 6.6 marked as not to be kept (nt), which each
// key is here: without the mark 17 and 10 us more. One token over 1,280 keys takes 10 us, a chain of dependent reads (offsets, page numbers, keys).
// Many rows (chunks, prompts): the matrix cores. 768, 257 and 512 queries over 20,280, 4,097 and 9,999 keys, 12 heads over 4 of 128: 140 to 143 us, 920 to
// 940 TFLOP/s, and 11 for the join of 42 MB of partial sums; a prompt of 6,912 tokens, 24 heads over 8, 338 us in all, where the kernel of whole offsets on
// the host (t2v_causal_fwd.hip), which deals tiles longest first and cuts fewer, takes 320; of 20,280 tokens 2,445 against 2,175, as
// there the workgroups of a die read other parts of more keys than its L2 holds.
// Every workgroup goes through the offsets and lengths of all sequences, 64 at a time: the chunks take 145 us among 64 sequences and 157 among 256, most of them
// idle.
// Mixtures run both at once, two workgroups a CU at head_dim 128 and three at 64, as many as registers and LDS let: 30 tokens beside chunks
// of 512 and 300, 804 MB: 148 us (as two launches, one after the other, 202).
#include <algorithm>

#include "t2v_causal_fwd_step.hpp"
#include "t2v_paged_kernels.h"

namespace t2v {

using namespace kern;

namespace {

constexpr int kFewRows = 32, kManyRows = 128;
constexpr float kNan = __builtin_nanf("");
// Time of a position of few rows against one of many. Four mixtures of tokens and chunks at head_dim 128, of 0.8, 0.95, 1.1, 1.25, 1.4 and 1.6: in the mean
// 3, 1, 7, 7, 14 and 23% slower than the best for each; five at 64, of 0.5, 0.65, 0.8, 0.95 and 1.1: 4, 6, 4, 1 and 2%.
constexpr float kFewWeight = 0.95f;
constexpr int kStage = 64;  // keys of an LDS stage of the kernel of 128 rows

typedef __attribute__((address_space(4))) const int32_t const_i32;  // read with scalar loads

// One tensor's pages: bytes between pages, tokens and heads.
struct Rows {
  const char* base;
  int64_t head;
  uint32_t page, token;
};
struct PagesView {
  Rows k, v;
  const_i32* table;
  const_i32* lengths;
  int64_t table_stride;
  int pages, shift, room;
};

// The first piece of the tile that a workgroup cuts, for the join. Pieces 1, 2, .. are those of the line's next shares.
struct PagedDesc {
  int64_t q0, first, next;  // first and second piece's place in the partial results, in floats
  int lq, row0, head, pieces, rows;
};

struct PagedArgs {
  const bf16* q;
  int64_t q_stride;
  const_i32* cu;
  int64_t tokens;
  PagesView c;
  PagedRule few, many;
  float weight;  // time of a position of few rows against one of many
  int nseq, heads, kv_heads;
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

// The kernel's arguments, read again by scalar loads where they are needed: all of them kept in scalar registers would leave too few
// to the loops.
typedef __attribute__((address_space(4))) const void const_void;
T2V_DEV const PagedArgs& arguments() {
  uint64_t p = (uint64_t)(__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(p));
  return *(const PagedArgs*)((const_void*)(p));
}

T2V_DEV PagedSeq seq_at(const PagedArgs& a, int s) {
  return paged_seq(a.cu[s], a.cu[s + 1], a.c.lengths[s], a.tokens, a.c.room);
}

// Sum over a wave's lanes up to this one, by moves between neighbouring lanes and rows of 16.
T2V_DEV int64_t wave_scan(int64_t x) {
  auto add = [&](auto ctrl, auto rows) {
    const uint64_t u = static_cast<uint64_t>(x);
    const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    x += static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(lo));
  };
  using All = std::integral_constant<int, 0xF>;
  add(std::integral_constant<int, 0x111>{}, All{});                                 // row_shr:1, 2, 4, 8
  add(std::integral_constant<int, 0x112>{}, All{});
  add(std::integral_constant<int, 0x114>{}, All{});
  add(std::integral_constant<int, 0x118>{}, All{});
  add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});    // row_bcast:15 into rows 1 and 3
  add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});    // row_bcast:31 into rows 2 and 3
  return x;
}

// This workgroup's line and its share of it: positions from .. to - 1, the first of which lies in key head `head` of sequence
// `seq`, whose interval begins at `at`.
struct Walk {
  bool many;
  int share, shares, n_few, head, seq;
  int64_t at, from, to, length;
  int period;  // keys of a share, 2^31 - 1 at most
};

// Each wave works it out by itself: costs of 64 sequences at a time, their sums over the lanes, and a search. (Offsets or lengths that
// something changes meanwhile may be found nowhere: then this workgroup does no work.)
T2V_DEV Walk find_share(const PagedArgs& a, int lane) {
  const int* cu = (const int*)(a.cu);
  const int* lengths = (const int*)(a.c.lengths);
  const PagedRule rules[2] = {a.few, a.many};
  int64_t cost[2], upto[2], sum[2] = {0, 0};  // cost: of one key head
  auto costs = [&](int s0) {  // of sequence s0 + lane on either line, and with all key heads of those up to it from s0 on
    const int s = s0 + lane;
    PagedSeq seq = {0, 0, 0, false};
    const bool real = s < a.nseq;
    if (real) seq = paged_seq(cu[s], cu[s + 1], lengths[s], a.tokens, a.c.room);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      cost[i] = real ? paged_cost(rules[i], paged_tiles(rules[i], seq)) : 0;
      upto[i] = wave_scan(cost[i] * a.kv_heads);
    }
  };
  for (int s0 = 0; s0 < a.nseq; s0 += 64) {
    costs(s0);
#pragma unroll
    for (int i = 0; i < 2; ++i) sum[i] = paged_add(sum[i], lane_of(upto[i], 63));
  }
  const int groups = gridDim.x, n_many = uniform(paged_many(groups, sum[0], sum[1], a.weight));
  const PagedRole role = paged_role(blockIdx.x, groups, n_many);
  const int64_t total = role.many ? paged_line(sum[1], sum[0]) : paged_line(sum[0], sum[1]);
  Walk w;
  w.many = role.many;
  w.n_few = groups - n_many;
  const PagedShares shares = paged_shares(role.many ? a.many : a.few, total, role.many ? n_many : groups - n_many, groups);
  w.share = role.x * shares.each + role.i;
  w.shares = shares.dies * shares.each;
  w.length = shares.length;
  w.period = static_cast<int>(min(shares.length, (static_cast<int64_t>(1) << 39) - 1) >> 8);
  w.from = w.share * w.length;
  w.to = role.i < shares.each ? min(total, w.from + w.length) : w.from;
  w.head = w.seq = 0;
  w.at = 0;
  if (w.from >= w.to) return w;
  int64_t base = 0;
  int s0 = 0;
  if (a.nseq > 64) {
    for (; s0 < a.nseq; s0 += 64) {
      costs(s0);
      const int64_t all = lane_of(role.many ? upto[1] : upto[0], 63);
      if (w.from < base + all) break;
      base += all;
    }
  }
  const int64_t rest = w.from - base, end = role.many ? upto[1] : upto[0], one = role.many ? cost[1] : cost[0];
  const int64_t begin = end - one * a.kv_heads;
  const uint64_t found = __ballot(rest >= begin && rest < end);
  if (found == 0) {
    w.to = w.from;
    return w;
  }
  const int at = __builtin_ctzll(found);
  const int64_t first = lane_of(begin, at), head_cost = lane_of(one, at);
  w.seq = s0 + at;
  w.head = uniform(paged_ratio(rest - first, head_cost));
  w.at = base + first + w.head * head_cost;
  return w;
}

// Partial results of a share's two slots: those of the line of few rows come first.
template <int D>
T2V_DEV int64_t slot_floats(const Walk& w, int rows) {
  return (w.many ? static_cast<int64_t>(w.n_few) * 2 * kFewRows * (D + 2) : 0) + static_cast<int64_t>(w.share) * 2 * rows * (D + 2);
}

// Runs f(sequence's number, sequence, its tiles, head, piece) for every piece of this workgroup's share, and leaves its
// descriptor.
template <int D, typename F>
T2V_DEV void for_pieces(Walk& w, F&& f) {
  bool begun = false;
  while (w.from < w.to && w.seq < arguments().nseq) {
    const PagedArgs& a = arguments();
    const PagedRule rule = w.many ? a.many : a.few;
    const PagedSeq s = seq_at(a, w.seq);
    const PagedTiles t = paged_tiles(rule, s);
    const int64_t cost = paged_cost(rule, t);
    if (w.from < w.at + cost) {
      int tile = paged_tile_at(rule, t, w.from - w.at);
      for (; tile < t.tiles && w.from < w.to; ++tile) {
        const int64_t at = w.at + paged_before(rule, t, tile), end = min(w.to, w.at + paged_before(rule, t, tile + 1));
        PagedPiece p;
        if (paged_piece(rule, s, t, tile, at, w.from, end, w.length, w.share, &p)) {
          if (p.pieces > 1) {
            begun = true;
            const int64_t place = slot_floats<D>(w, rule.tile), slot = static_cast<int64_t>(rule.tile) * (D + 2);
            if (threadIdx.x == 0)
              arguments().desc[blockIdx.x] = {s.q0, place + slot, place + 2 * slot, s.lq, tile * rule.tile, w.head, min(p.pieces, w.shares - w.share), rule.tile};
          }
          f(w.seq, s, t, w.head, p);
        }
        w.from = end;
      }
    }
    w.at += cost;
    if (cost == 0 || ++w.head == a.kv_heads) {
      w.head = 0;
      ++w.seq;
    }
  }
  if (!begun && threadIdx.x == 0) arguments().desc[blockIdx.x].pieces = 0;
}

// Row r of a tile: where it is in [T, H, D] tensors, and the last key that it sees. Rows behind the last repeat it.
T2V_DEV LaneRow row_of(const PagedArgs& a, const PagedSeq& s, const PagedTiles& t, int head, int row) {
  const PackedRow pr = packed_row(min(row, t.rows - 1), a.few.group);
  return {row < t.rows, pr.query + (s.lk - s.lq), head * a.few.group + pr.head, s.q0 + pr.query};
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

// What the loops read of a sequence's pages, for one key head. BIG: pages of 64 keys or more, so that all keys of a
// step or a stage lie in one; else 16 neighbouring keys do.
struct HeadPages {
  const_i32* table;
  const char *k, *v;
  uint32_t k_page, k_token, v_page, v_token;
  int pages, shift, lk;
};
T2V_DEV HeadPages head_pages(const PagedArgs& a, int seq, int head, int lk) {
  const PagesView& c = a.c;
  return {c.table + seq * c.table_stride, c.k.base + head * c.k.head, c.v.base + head * c.v.head, c.k.page, c.k.token, c.v.page,
          c.v.token, c.pages, c.shift, lk};
}

// Number of the page that holds key `key` (or the last key, if that comes first).
T2V_DEV int page_of(const HeadPages& c, int key) { return c.table[min(key, c.lk - 1) >> c.shift]; }

// Where the keys from `key` on lie: addresses of its K and V (uniform), and how many rows behind it may be read. A page outside the cache
// is the row of NaN, for the key and all behind it.
struct Block {
  const char *k, *v;
  int last;
};
T2V_DEV Block block_at(const HeadPages& c, int id, int key) {
  const int first = min(key, c.lk - 1);
  const bool ok = static_cast<unsigned>(id) < static_cast<unsigned>(c.pages);
  const uint32_t row = first & ((1 << c.shift) - 1);
  const uint64_t page = static_cast<uint32_t>(id);
  const char* nan = reinterpret_cast<const char*>(nan_row);
  return {ok ? c.k + (page * c.k_page + row * c.k_token) : nan, ok ? c.v + (page * c.v_page + row * c.v_token) : nan,
          ok && key < c.lk ? c.lk - 1 - key : 0};
}

#if T2V_CHECKED
// Whether row r behind key `key` may be read; a row that may not is replaced by NaN.
T2V_DEV bool check_key(const HeadPages& c, int key, int r) { return check_row(min(key, c.lk - 1) + r, c.lk); }
#endif

// ------------------------------------------------------------------ few rows: single tokens

// As dma_lds16_s, for bytes that nothing reads again: they need not stay in the caches, which serve 6.6 TB/s of them in place of 6.0.
T2V_DEV void dma_lds16_once(const void* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff), "s"(uniform_ptr(sbase)), "{m0}"(lds) : "memory");
}

// Copy of 32 keys by one wave into swizzled tiles of K and V; instruction j covers RPI rows. Its swizzle differs from instruction
// 0's by a constant.
template <int D, bool BIG>
struct StepDma {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NJ = 32 / RPI;
  static constexpr int NB = BIG ? 1 : 2, PER = NJ / NB;  // blocks of keys that lie together, and their instructions
  int r0;
  uint32_t chunk0;
  T2V_DEV explicit StepDma(int lane) : r0(lane / CPR), chunk0(static_cast<uint32_t>((lane % CPR) ^ swz<D>(lane / CPR))) {}
  T2V_DEV uint32_t col(int j) const { return (chunk0 ^ static_cast<uint32_t>(swz<D>(RPI * j))) * 16; }
  T2V_DEV void find(int (&ids)[NB], const HeadPages& c, int key0) const {
#pragma unroll
    for (int h = 0; h < NB; ++h) ids[h] = page_of(c, key0 + 16 * h);
  }
  T2V_DEV void copy(uint32_t k_tile, uint32_t v_tile, const HeadPages& c, const int (&ids)[NB], int key0) const {
    Block b[NB];
#pragma unroll
    for (int h = 0; h < NB; ++h) b[h] = block_at(c, ids[h], key0 + 16 * h);
    bool whole = !T2V_CHECKED;
#pragma unroll
    for (int h = 0; h < NB; ++h) whole = whole && b[h].last >= RPI * PER - 1;
    if (whole) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t token = t ? c.v_token : c.k_token, tile = t ? v_tile : k_tile, row = static_cast<uint32_t>(r0) * token;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          dma_lds16_once((t ? b[j / PER].v : b[j / PER].k) + static_cast<uint64_t>(RPI * (j % PER)) * token, row + col(j), tile + j * 1024);
      }
      return;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t token = t ? c.v_token : c.k_token, tile = t ? v_tile : k_tile;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const Block& at = b[j / PER];
        const int r = min(r0 + RPI * (j % PER), at.last);
#if T2V_CHECKED
        if (!check_key(c, key0 + 16 * (j / PER), r)) {
          dma_lds16_once(nan_row, col(j), tile + j * 1024);
          continue;
        }
#endif
        dma_lds16_once(t ? at.v : at.k, static_cast<uint32_t>(r) * token + col(j), tile + j * 1024);
      }
    }
  }
};

// A tile of at most 32 packed rows, which the workgroup's four waves all hold: they take every fourth 32-key step, each through an LDS
// buffer of its own, which is filled again as soon as its step's operands are in registers; so nothing but its own copies holds a wave
// up. The waves' sums meet in LDS at the end.
template <int D, bool BIG>
T2V_DEV void few_pieces(Walk& w, bf16* lds, float (&sM)[4][kFewRows], float (&sL)[4][kFewRows]) {
  using Dma = StepDma<D, BIG>;
  constexpr int KK = D / 16, DB = D / 32, R = kFewRows;
  constexpr int kTile = 32 * D;  // elements of a step's K or V
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = uniform(tid >> 6);
  const int G = lane >> 5, l32 = lane & 31;
  bf16* const buf = lds + wave * (2 * kTile);
  const Dma dma(lane);
  const uint32_t k_tile = lds_addr(buf), v_tile = k_tile + 2 * kTile;
  const uint32_t ko = k_tile + opnd_lane_off<D>(lane);
  const uint32_t vo0 = v_tile + rows_lane_off<D>(lane, 0), vo1 = v_tile + rows_lane_off<D>(lane, 1);
  for_pieces<D>(w, [&](int seq, const PagedSeq& s, const PagedTiles& t, int head, const PagedPiece& p) {
    const PagedArgs& a = arguments();
    const int row0 = p.tile * R;
    const LaneRow me = row_of(a, s, t, head, row0 + l32);
    const int lim_lo = __builtin_amdgcn_readlane(me.lim, 0);
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    float m_run = -kInf, l_run = 0.0f;
    const int nsteps = (p.end - p.begin + 31) / 32;
    if (wave < nsteps) {
      const HeadPages pages = head_pages(a, seq, head, s.lk);
      const float scale = a.scale;
      int ids[Dma::NB];
      auto fetch = [&](int n) {
        dma.copy(k_tile, v_tile, pages, ids, p.begin + n * 32);
        if (n + 4 < nsteps) dma.find(ids, pages, p.begin + (n + 4) * 32);
      };
      dma.find(ids, pages, p.begin + wave * 32);
      fetch(wave);
      bf16x8 qop[KK];
      load_queries(a, a.q + me.token * a.q_stride + static_cast<int64_t>(me.head) * D, me.ok, G, qop, KK);
      // Steps that all rows see whole, then the others.
      int n = wave;
      auto arrived = [&] {
        wait_vmcnt0();
        asm volatile("" ::: "memory");
      };
      auto next = [&] {
        if (n + 4 < nsteps) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this step's operands have left the buffer
          fetch(n + 4);
        }
      };
      for (; n < nsteps && p.begin + n * 32 + 31 <= lim_lo; n += 4) {
        arrived();
        fwd_step<D, false, true>(ko, vo0, vo1, 0, 0, scale, qop, o, m_run, l_run, lane, next);
      }
#pragma unroll 1
      for (; n < nsteps; n += 4) {
        arrived();
        fwd_step<D, true>(ko, vo0, vo1, 0, me.lim - (p.begin + n * 32), scale, qop, o, m_run, l_run, lane);
        next();  // not before: the step may read its values again
      }
    }

    // The waves' sums, unnormalised and each with its own reference, in fp32: wave w's in its buffers.
    const float lt = half_sum(l_run);
    float* mine = reinterpret_cast<float*>(buf);
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
      for (int i = 1; i < 4; ++i) m = max_nan(m, sM[i][r]);
      const float ref = m == -kInf ? 0.0f : m;
      float l = 0.0f, x[C];
#pragma unroll
      for (int e = 0; e < C; ++e) x[e] = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = __builtin_amdgcn_exp2f(sM[i][r] - ref);
        l = fmaf(f, sL[i][r], l);
        const float* src = reinterpret_cast<const float*>(lds + i * (2 * kTile)) + r * D + col;
#pragma unroll
        for (int e = 0; e < C; ++e) x[e] = fmaf(f, src[e], x[e]);
      }
      if (p.slot >= 0) {
        float* po = a.partial + slot_floats<D>(w, R) + (p.slot & 1) * (R * (D + 2));
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
          bf16x8 y;
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = static_cast<bf16>(x[e + i] * inv);
          *reinterpret_cast<bf16x8*>(op + e) = y;
        }
        if (col == 0)
          a.lse[static_cast<int64_t>(row.head) * a.tokens + row.token] = s.bad ? kNan : (m + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
    __syncthreads();  // before the next piece's copies over the sums
  });
}

// ------------------------------------------------------------------ many rows: chunks and prompts

// Copy of a stage of 64 keys by a workgroup into swizzled tiles of K and V: wave w's instruction j covers RPI rows from row RPI (w + NW j) on,
// which lie in one block of 16.
template <int D, int NT, bool BIG>
struct StageDma {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NW = NT / 64, NJ = kStage / RPI / NW;
  static constexpr int NB = BIG ? 1 : NJ;
  static_assert((RPI * NW) % 16 == 0, "a lane's swizzled chunk must not depend on the instruction");
  int wave, r;  // r: this lane's row of its block of 16, or (BIG) of the stage in instruction 0
  uint32_t col;
  T2V_DEV explicit StageDma(int tid) {
    wave = uniform(tid >> 6);
    const int row = RPI * wave + (tid & 63) / CPR;
    r = BIG ? row : row & 15;
    col = static_cast<uint32_t>((((tid & 63) % CPR) ^ swz<D>(row)) * 16);
  }
  // First key of what lies together in instruction j.
  T2V_DEV int block(int j) const { return BIG ? 0 : (RPI * (wave + NW * j)) & ~15; }
  T2V_DEV void find(int (&ids)[NB], const HeadPages& c, int key0) const {
#pragma unroll
    for (int j = 0; j < NB; ++j) ids[j] = page_of(c, key0 + block(j));
  }
  T2V_DEV void copy(bf16* k_tile, bf16* v_tile, const HeadPages& c, const int (&ids)[NB], int key0) const {
    Block b[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) b[j] = block_at(c, ids[j], key0 + block(j));
    bool whole = !T2V_CHECKED;
#pragma unroll
    for (int j = 0; j < NB; ++j) whole = whole && b[j].last >= (BIG ? kStage : 16) - 1;
    if (whole) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t token = t ? c.v_token : c.k_token, lds = lds_addr(t ? v_tile : k_tile) + wave * 1024;
        const uint32_t off = static_cast<uint32_t>(r) * token + col;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          dma_lds16_s((t ? b[BIG ? 0 : j].v : b[BIG ? 0 : j].k) + static_cast<uint64_t>(BIG ? RPI * NW * j : 0) * token, off,
                      lds + j * NW * 1024);
      }
      return;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t token = t ? c.v_token : c.k_token, lds = lds_addr(t ? v_tile : k_tile) + wave * 1024;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const Block& at = b[BIG ? 0 : j];
        const int row = min(r + (BIG ? RPI * NW * j : 0), at.last);
#if T2V_CHECKED
        if (!check_key(c, key0 + block(j), row)) {
          dma_lds16_s(nan_row, col, lds + j * NW * 1024);
          continue;
        }
#endif
        dma_lds16_s(t ? at.v : at.k, static_cast<uint32_t>(row) * token + col, lds + j * NW * 1024);
      }
    }
  }
};

// Stage of a piece that comes first, where `clock` keys of the share have been gone through: key k has its turn at clock k modulo the share's
// keys (or the tile's, if it has fewer).
T2V_DEV int first_stage(const Walk& w, const PagedPiece& p, unsigned clock) {
  const unsigned begin = p.begin, period = min(w.period, p.n), at = clock % period;
  const unsigned key = at + (begin <= at ? 0 : (begin - at + period - 1) / period * period);
  return key < static_cast<unsigned>(p.end) ? static_cast<int>(key - begin) / kStage : 0;
}

// A tile of 128 packed rows, 32 to a wave; the workgroup stages 64 keys at a time for all of them, the next ones under the
// products of these.
template <int D, bool BIG>
T2V_DEV void many_pieces(Walk& w, bf16* lds) {
  constexpr int KK = D / 16, DB = D / 32, NT = 256, R = kManyRows;
  using Dma = StageDma<D, NT, BIG>;
  auto sK = [&](int b) { return lds + b * (kStage * D); };
  auto sV = [&](int b) { return lds + (2 + b) * (kStage * D); };
  const int tid = threadIdx.x;
  const int wave = uniform(tid >> 6);
  unsigned clock = 0;  // keys of the pieces so far, rounded up to stages
  for_pieces<D>(w, [&](int seq, const PagedSeq& s, const PagedTiles& t, int head, const PagedPiece& p) {
    const int lane = lane_again(), G = lane >> 5, l32 = lane & 31;
    const int row0 = p.tile * R + wave * 32;
    const bool wave_active = row0 < t.rows;
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = zero16();
    float m_run = -kInf, l_run = 0.0f;
    const int ntiles = (p.end - p.begin + kStage - 1) / kStage;
    if (ntiles > 0) {
      const PagedArgs& a = arguments();
      const LaneRow me = row_of(a, s, t, head, row0 + l32);
      const int lim = me.lim, lim_lo = __builtin_amdgcn_readlane(lim, 0), lim_hi = __builtin_amdgcn_readlane(lim, 31);
      const HeadPages pages = head_pages(a, seq, head, s.lk);
      const float scale = a.scale;
      const Dma dma(tid);
      // The stages are gone through from `first` on and around, for a key to have its turn at the same time in all of a die's workgroups, whose
      // pieces begin at other keys: what one reads from memory the others find in the die's L2 then.
      const int first = first_stage(w, p, clock);
      clock += ntiles * kStage;
      auto key_at = [&](int j) { return p.begin + (first + j < ntiles ? first + j : first + j - ntiles) * kStage; };
      int ids[Dma::NB];
      dma.find(ids, pages, key_at(0));
      dma.copy(sK(0), sV(0), pages, ids, key_at(0));
      if (ntiles > 1) dma.find(ids, pages, key_at(1));
      bf16x8 qop[KK];
      load_queries(a, a.q + me.token * a.q_stride + static_cast<int64_t>(me.head) * D, me.ok, G, qop, KK);
      const uint32_t ko = opnd_lane_off<D>(lane);
      const uint32_t vo0 = rows_lane_off<D>(lane, 0), vo1 = rows_lane_off<D>(lane, 1);
      wait_vmcnt0();
      __syncthreads();
      auto prefetch = [&](int j) {
        if (j + 1 < ntiles) {
          dma.copy(sK((j & 1) ^ 1), sV((j & 1) ^ 1), pages, ids, key_at(j + 1));
          if (j + 2 < ntiles) dma.find(ids, pages, key_at(j + 2));
        }
      };
      // Stages that all rows of this wave see whole (before key `full`), and the others, the tile's last: every wave passes ntiles barriers.
      const int full = wave_active ? p.begin + min(max(lim_lo + 1 - p.begin, 0) / kStage, ntiles) * kStage : p.begin;
      for (int j = 0; j < ntiles;) {
        for (; j < ntiles && key_at(j) < full; ++j) {
          const int b = j & 1;
          prefetch(j);
          const uint32_t kbase = lds_addr(sK(b)) + ko;
          const uint32_t vb0 = lds_addr(sV(b)) + vo0, vb1 = lds_addr(sV(b)) + vo1;
#pragma unroll
          for (int kb = 0; kb < kStage; kb += 32)
            fwd_step<D, false>(kbase, vb0, vb1, kb, 0, scale, qop, o, m_run, l_run, lane);
          wait_vmcnt0();
          __syncthreads();
        }
        for (; j < ntiles && key_at(j) >= full; ++j) {
          const int b = j & 1;
          const int key0 = key_at(j);
          prefetch(j);
          if (wave_active) {
            const uint32_t kbase = lds_addr(sK(b)) + ko;
            const uint32_t vb0 = lds_addr(sV(b)) + vo0, vb1 = lds_addr(sV(b)) + vo1;
#pragma unroll 1
            for (int kb = 0; kb < kStage && key0 + kb <= lim_hi; kb += 32)
              fwd_step<D, true>(kbase, vb0, vb1, kb, lim - key0 - kb, scale, qop, o, m_run, l_run, lane);
          }
          wait_vmcnt0();
          __syncthreads();
        }
      }
    }
    if (wave_active) {
      // Worked out again, rather than kept in registers through the loop.
      const PagedArgs& a = arguments();
      const int lane = lane_again(), G = lane >> 5, l32 = lane & 31;
      const LaneRow me = row_of(a, s, t, head, row0 + l32);
      const float lt = half_sum(l_run);
      if (p.slot >= 0) {  // one piece: unnormalised sums, reference and sum of each row
        float* po = a.partial + slot_floats<D>(w, R) + (p.slot & 1) * (R * (D + 2));
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
}

template <int D, bool BIG>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void paged_fwd_kernel(const PagedArgs) {
  __shared__ __attribute__((aligned(1024))) bf16 lds[4 * kStage * D];  // two stages of K and V, or a step of them for each wave
  __shared__ float sM[4][kFewRows], sL[4][kFewRows];
  const unsigned long long trace_t0 = arguments().trace != nullptr ? trace_clock() : 0ull;
  Walk w = find_share(arguments(), threadIdx.x & 63);
  if (w.many)
    many_pieces<D, BIG>(w, lds);
  else
    few_pieces<D, BIG>(w, lds, sM, sL);
  if (arguments().trace != nullptr) trace_end(arguments().trace, trace_t0, 0, blockIdx.x);
}

// ------------------------------------------------------------------ join

// Workgroups of a cut tile, in calls that can have tiles of many rows; of a tile of few rows, all but one return at once. The chunks above: 20 us with one, 11
// with four (10 with eight). 32 tokens take 5.1 us for the 4.8 with one; a chunk of 512 tokens, 24 heads over 8, 10.7 for 20.4.
constexpr int kJoinBlocks = 4;
constexpr int kJoinAhead = 4;  // pieces of a row in flight (a token over 100,000 keys: 5.6 us; one after the other, by 16 lanes, 24; eight: 5.2, mixtures 10 for 7)

struct JoinArgs {
  const float* partial;
  const PagedDesc* desc;
  int blocks, heads, group;  // workgroups of a descriptor
  int64_t tokens;
  bf16* out;
  float* lse;
};

// Joins the pieces of the tile that a workgroup begins: with the largest reference m of a row, out = sum_p 2^(m_p - m) O_p / l,
// l = sum_p 2^(m_p - m) l_p, in piece order. D / 8 lanes hold a row, eight columns each. Of a tile with fewer rows than a workgroup holds, several groups
// of lanes take parts of the pieces, whose sums meet in LDS, in order. Every row sees keys: a tile is cut where its last row sees twice the shortest piece, 256
// keys, or more, and has 128 queries at most.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const JoinArgs a) {
  constexpr int LPR = D / 8, RPB = kThreads / LPR;
  __shared__ __attribute__((aligned(16))) float part_x[RPB][D];
  __shared__ float part_l[RPB];
  const PagedDesc it = a.desc[blockIdx.x / a.blocks];
  if (it.pieces == 0) return;
  const int sub = threadIdx.x % LPR, col = sub * 8, group = threadIdx.x / LPR, block = blockIdx.x % a.blocks;
  const int64_t share = static_cast<int64_t>(it.rows) * 2 * (D + 2);
  auto piece = [&](int i) { return a.partial + (i == 0 ? it.first : it.next + (i - 1) * share); };
  const int rows = min(it.rows, it.lq * a.group - it.row0);
  int parts = 1;
  while (2 * parts * rows <= RPB) parts *= 2;
  const int per_part = (it.pieces + parts - 1) / parts, held = RPB / parts;  // rows at a time
  if (parts > 1 && block > 0) return;
  for (int r0 = parts > 1 ? 0 : block * RPB; r0 < rows; r0 += a.blocks * RPB) {  // all threads alike
    const int r = r0 + group % held, part = group / held;
    const bool real = r < rows;
    const int begin = part * per_part, end = real ? min(begin + per_part, it.pieces) : begin;
    const int mo = it.rows * D + 2 * r, xo = r * D + col;
    float m = -kInf;
    for (int i = real ? sub : it.pieces; i < it.pieces; i += LPR) m = max_nan(m, piece(i)[mo]);
#pragma unroll
    for (int off = LPR / 2; off > 0; off >>= 1) m = max_nan(m, __shfl_xor(m, off, LPR));
    const float ref = m == -kInf ? 0.0f : m;
    float l = 0.0f;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = x;
    for (int i0 = begin; i0 < end; i0 += kJoinAhead) {
      f32x4 u[kJoinAhead], v[kJoinAhead];
      float w[kJoinAhead], lw[kJoinAhead];
#pragma unroll
      for (int e = 0; e < kJoinAhead; ++e) {
        const float* src = piece(min(i0 + e, end - 1));
        u[e] = *reinterpret_cast<const f32x4*>(src + xo);
        v[e] = *reinterpret_cast<const f32x4*>(src + xo + 4);
        w[e] = src[mo];
        lw[e] = src[mo + 1];
      }
#pragma unroll
      for (int e = 0; e < kJoinAhead; ++e) {
        if (i0 + e >= end) break;
        const float f = __builtin_amdgcn_exp2f(w[e] - ref);
        l = fmaf(f, lw[e], l);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          x[c] = fmaf(f, u[e][c], x[c]);
          y[c] = fmaf(f, v[e][c], y[c]);
        }
      }
    }
    if (parts > 1) {
      *reinterpret_cast<f32x4*>(&part_x[group][col]) = x;
      *reinterpret_cast<f32x4*>(&part_x[group][col + 4]) = y;
      if (sub == 0) part_l[group] = l;
      __syncthreads();
      for (int g = group + held; part == 0 && g < RPB; g += held) {
        l += part_l[g];
        x += *reinterpret_cast<const f32x4*>(&part_x[g][col]);
        y += *reinterpret_cast<const f32x4*>(&part_x[g][col + 4]);
      }
    }
    if (!real || part > 0) continue;
    const PackedRow pr = packed_row(it.row0 + r, a.group);
    const float inv = 1.0f / l;
    const int64_t token = it.q0 + pr.query;
    const int head = it.head * a.group + pr.head;
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = static_cast<bf16>(x[e] * inv);
      o[4 + e] = static_cast<bf16>(y[e] * inv);
    }
    *reinterpret_cast<bf16x8*>(a.out + (token * a.heads + head) * D + col) = o;
    if (col == 0) a.lse[static_cast<int64_t>(head) * a.tokens + token] = (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// ------------------------------------------------------------------ launches

Rows rows_of(const void* base, const int64_t (&strides)[3]) {
  return {static_cast<const char*>(base), 2 * strides[2], static_cast<uint32_t>(2 * strides[0]), static_cast<uint32_t>(2 * strides[1])};
}

int64_t desc_bytes(int groups) { return (static_cast<int64_t>(groups) * sizeof(PagedDesc) + 255) / 256 * 256; }

}  // namespace

int paged_few_rows() { return kFewRows; }
int paged_many_rows() { return kManyRows; }
int paged_least_share() { return 128; }
int paged_groups(int head_dim, int ncu) { return std::max(1, ncu) * (head_dim == 64 ? 3 : 2); }
int64_t paged_workspace(int groups, bool only_few, int head_dim) {
  return desc_bytes(groups) + 2 * static_cast<int64_t>(groups) * (only_few ? kFewRows : kManyRows) * (head_dim + 2) * 4;
}

hipError_t launch_paged_fwd(const PagedCall& c, int groups, void* ws, hipStream_t s) {
  PagedArgs a{};
  const t2v_pages& g = c.cache;
  const int group = c.heads / g.kv_heads;
  a.q = static_cast<const bf16*>(c.q);
  a.q_stride = c.q_stride;
  a.cu = (const_i32*)(c.cu);
  a.tokens = c.tokens;
  a.c.k = rows_of(g.k, g.k_strides);
  a.c.v = rows_of(g.v, g.v_strides);
  a.c.table = (const_i32*)(g.table);
  a.c.lengths = (const_i32*)(g.lengths);
  a.c.table_stride = g.table_stride;
  a.c.pages = static_cast<int>(g.pages);
  a.c.shift = __builtin_ctz(g.page_size);
  a.c.room = g.width * g.page_size;
  // Cuts are at multiples of the four waves' steps, or of a stage. A tile's fixed part is 256 keys: with 64, 32 tokens over 31 to 20,280 keys take 159 us
  // for 153 (graphs replayed), with 1,024 158, and 60 beside a chunk of 700, 30 heads of 64 over 10, 168 for 160. Shares have 128 keys at least: with 512, 64
  // tokens over 300 take 26 us for 23, and longer ones as long.
  a.few = paged_rule(group, kFewRows, 128, 128, 256, paged_least_share(), kPagedFew, kFewRows);
  a.many = paged_rule(group, kManyRows, kStage, 128, 256, paged_least_share(), kPagedMany, kFewRows);
  a.weight = kFewWeight;
  a.nseq = g.nseq;
  a.heads = c.heads;
  a.kv_heads = g.kv_heads;
  // A negative scale turns the sign of Q (so that the largest scaled score is that of the largest product), a scale of 0 clears it.
  a.scale = c.scale == 0.0f ? 1.0f : fabsf(c.scale) * kLog2e;
  a.qkeep = c.scale == 0.0f ? 0u : ~0u;
  a.qflip = c.scale < 0.0f ? 0x80008000u : 0u;
  a.out = static_cast<bf16*>(c.out);
  a.lse = c.lse;
  a.desc = static_cast<PagedDesc*>(ws);
  a.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + desc_bytes(groups));
  a.trace = c.trace;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, s, a); };
  if (g.page_size >= kStage)
    g.head_dim == 128 ? launch(paged_fwd_kernel<128, true>) : launch(paged_fwd_kernel<64, true>);
  else
    g.head_dim == 128 ? launch(paged_fwd_kernel<128, false>) : launch(paged_fwd_kernel<64, false>);
  return hipGetLastError();
}

hipError_t launch_paged_join(const PagedCall& c, int groups, void* ws, hipStream_t s) {
  const int d = c.cache.head_dim, group = c.heads / c.cache.kv_heads;
  const int blocks = paged_join_blocks(c.tokens * group, kFewRows, kJoinBlocks);
  const JoinArgs a{reinterpret_cast<const float*>(static_cast<char*>(ws) + desc_bytes(groups)), static_cast<const PagedDesc*>(ws), blocks,
                   c.heads, group, c.tokens, static_cast<bf16*>(c.out), c.lse};
  if (d == 128)
    hipLaunchKernelGGL((paged_join_kernel<128>), dim3(groups * blocks), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((paged_join_kernel<64>), dim3(groups * blocks), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

#if T2V_CHECKED
hipError_t paged_fwd_check_take(unsigned int* rec, unsigned int canary) { return kern::check_take_here(rec, canary); }
#endif
}  // namespace t2v
