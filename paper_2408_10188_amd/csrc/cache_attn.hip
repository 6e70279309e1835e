// Attention of new tokens over a paged key-value cache: every K and V row is read once for the handful of query rows that
// share its KV head, so the memory rate bounds it (28/4 heads, one token: 7 of the 16 columns of a matrix instruction, 7 flops a byte).
//
// Work.  The (token, head) pairs of a KV head's new rows are one list, as in the forward kernel; groups of kRows of it are
// stationary, 16, 32 or 48 of them.  A pair of (sequence, KV head, group) has the sequence's keys in tiles.  The tiles of all pairs are one sequence that is cut
// into as many equal ranges as there are workgroups (or half as many, see pick_cut), whatever the lengths are: a workgroup goes through the segments
// of pairs in its range.  A pair inside one range is finished there; at most the first and the last segment of a range are
// parts of pairs that others share: their (O, maximum, sum) goes to the workspace and a second launch joins them.  The lengths are on the device only,
// so each workgroup adds up the tiles of all sequences for itself.
//
// Wavefronts.  Those of a workgroup take different keys, 32 (f32: 16) a step, and meet when a segment ends, so the loop has no barrier: each
// has LDS of its own for K and V of one step, and asks for the next step's K as soon as it has read this one's, and so for V.  The copies are asynchronous, and
// their waits written out, as in the forward (loads into registers were moved together, ahead of their waits, by the compiler: 69 instead of 64 us for 64
// ragged sequences).  S^T = K . Q^T, O^T += V^T . P^T: the 16 keys of a block are dealt to the contraction
// slots so that the accumulators of S^T are B operands as they are, and a lane's V pieces (8 elements of d of the 8 keys of its
// slots) become the A operands of 8 products by exchanging halves of registers.
//
// Teams.  Where a sequence has more rows than a group takes, workgroups on one XCD take a group each and read the same keys at the same time (Teams).
//
// Measured, 28/4 heads, one token, both launches: 203 tokens 7.2 us (a chain: lengths, pages and Q, K and V, the results), 256K tokens 87 us, of which the loop reads
// 6.9 TB/s (a plain read of that size 7.1), 64 sequences of 150 to 16384 tokens 63.8 us.  The compiler keeps 66 to 97 scalars of a kernel in lanes of vector registers (no vector
// register goes to memory); what that costs has not been measured.
#include <algorithm>
#include <type_traits>

#include "mfma_tiles.h"
#include "paged.h"

namespace mmsp {
namespace {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

constexpr int kMaxGroups = 1024;                        // workgroups of a launch
constexpr int kMaxTeam = 8;                             // .. that read the same keys

struct Partial {
  u32x2* parts;                                         // [n_rows][Hq] the block that has the first tile, and (how many teams have some) << 8 | row of its group
  float* m; float* l;                                   // [2 W][kRows]
  float* o;                                             // [2 W][kRows][d]
};

// Workgroups come in teams of `size` that read the same keys at the same time for different groups of rows, so that memory is read once and the others find the keys in
// their L2: blocks b and b + 8 are on the same XCD.  rows: those of a team, size * kRows.
struct Teams { int count, alone, size; FastDiv rows; };   // alone: for teams of one, as many as have a CU to themselves; else all
struct Place { int team, member; };
__device__ __forceinline__ Place place_of(const Teams& t, int block) {
  const int i = block >> 3, q = i / t.size;
  return {(block & 7) + 8 * q, i - q * t.size};
}
__device__ __forceinline__ int block_of(const Teams& t, int team, int member) { return (team & 7) + 8 * ((team >> 3) * t.size + member); }

// Rounds in which a team takes the rows of a KV head's list, and tiles of each of these pairs.
struct PairShape { int rounds, tiles; };
__device__ __forceinline__ PairShape pairs_of(const CacheAttnArgs& a, const Teams& teams, const SeqRows& r, int tile_bits) {
  PairShape p;
  p.rounds = (int)(((uint32_t)r.count * a.group + teams.rows.d - 1) / teams.rows);
  p.tiles = max(1, (r.length + (1 << tile_bits) - 1) >> tile_bits);   // rows that see nothing have a tile too: someone has to say so
  return p;
}

// kN numbers, 4 or 8, to `at` and on, as bf16 or fp32.
template <bool kBf16, int kN>
__device__ __forceinline__ void store_row(void* to, int64_t at, const float (&x)[kN]) {
  static_assert(kN == 4 || kN == 8, "whole pieces of 4");
  if constexpr (kBf16) {
    uint32_t w[kN / 2];
#pragma unroll
    for (int e = 0; e < kN / 2; ++e) w[e] = pack2(x[2 * e], x[2 * e + 1]);
    uint16_t* const p = reinterpret_cast<uint16_t*>(to) + at;
    if constexpr (kN == 8) *reinterpret_cast<u32x4*>(p) = mk4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
  } else {
    float* const p = reinterpret_cast<float*>(to) + at;
#pragma unroll
    for (int e = 0; e < kN; e += 4) *reinterpret_cast<f32x4*>(p + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  }
}

// Asynchronous copy of 64 x 16 bytes to LDS (see dma16).  What is read once goes past the caches: 7.1 TB/s in a large plain read where the default policy reaches
// 6.2.  What a team shares does not (two members, 16 x 20000 keys: 149 instead of 173 us).
template <bool kShared>
__device__ __forceinline__ void copy_piece(const char* base, uint32_t offset, const void* lds_array, int byte_offset) {
  const uint32_t lds = lds_address(lds_array) + (uint32_t)byte_offset;
  if constexpr (kShared) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(lds), "v"(offset), "s"(base) : "memory");
}
// Until all but the last n copies have landed; until all LDS reads have returned.
template <int kN>
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kN) : "memory"); }
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// A word of V (two bf16 numbers or one f32) with zeros in the place of infinities and NaN.
template <bool kBf16>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
  if constexpr (kBf16) return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
  else return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
}

// Tiles of a workgroup's range: workgroup w has tiles [w * each, (w + 1) * each) of `total`.  (The host has made sure that there are at most 2^30.)
__device__ __forceinline__ int tiles_each(int total, int n_teams) { return max(1, (int)(((uint32_t)total + n_teams - 1) / (uint32_t)n_teams)); }

// A sum that the host has ruled out comes from a cu_new that is not ascending: no tile is taken.
__device__ __forceinline__ int checked_total(int total) { return total < 0 || total > 1 << 30 ? 0 : total; }

// How the tiles of a call are shared out: keys of a tile, as a logarithm; teams, all of them, two workgroups a CU, or only those that have a CU to themselves (the others
// leave at once); and how many tiles a pair counts for beside its own, where ranges hold several pairs, each of which costs some 2 us to begin and to end.
struct Cut { int bits, teams, extra; };
constexpr int fewest_bits(bool bf16) { return bf16 ? 7 : 6; }
constexpr int kExtra = 2;
// With many pairs: ranges of the smallest tiles for two workgroups a CU, one of which computes while the other begins or ends a pair.  28/4 heads, 200 sequences of 50 to 8000
// and up to four new tokens, us with tiles of 256 keys, no extra tiles / 256 and one / 128 and two / three: 127 / 114 / 112 / 115; 70 of 100 to 16000 and one: 89.7 / 84.1 /
// 84.6 / 85.2; 200 of 2000 and one: 134.6 / 133.1 / 135.1 / 136.1.
__device__ __forceinline__ Cut usual_cut(int fewest, const Teams& teams) { return {fewest, teams.count, kExtra}; }
// Counted in keys that a CU goes through, the cheapest of
//   alone   one tile a workgroup, one workgroup a CU,
//   split   ranges of several of the smallest tiles, one workgroup a CU (teams of several: two; one costs those with idle members up to 15 %),
//   shared  one tile a workgroup, two a CU, which get in each other's way (9/8).
// (The numbers here, in usual_cut and in plan_of are of 28/4 heads in bf16 unless they say otherwise; the rules count keys, rows and CUs, but other heads and f32 have not been measured against them.)
// 28/4 heads, us with tiles of 128 / 256 / 512 / 1024 keys for two workgroups a CU, and so picked: 20000 keys and three new tokens 20.1 / 20.0 / 17.6 / 22.4, 17.9 (alone);
// 8 sequences of 5003 and three 28.4 / 27.6 / 27.6 / 24.1, 23.9 (split); 16 of 5003 and five 40.5 / 45.4 / 47.6 / 47.3, 39.8 (split); 64 of 150 to 16384 and one
// 66.8 / 67.1 / 65.7 / -, 64.6 (split; pairs without extra tiles 67.6); 33 of 100 to 3000 and up to six 29.6 / 24.4 / 28.0 / 28.8, 25.3 (shared).
// tiles(bits): those of this lane's sequence; pairs: its pairs.
template <int kFewest, class Tiles>
__device__ __forceinline__ Cut pick_cut(Tiles tiles, int pairs, int n_seqs, const Teams& teams) {
  constexpr int kMost = 10, kNever = 1 << 30;
  int n[kMost - kFewest + 2];
#pragma unroll
  for (int b = kFewest; b <= kMost; ++b) n[b - kFewest] = min(tiles(b), 1 << 24);   // 64 of them stay below 2^31
  int& all_pairs = n[kMost - kFewest + 1];
  all_pairs = min(pairs, 1 << 22);
#pragma unroll 1
  for (int w = 1; w < n_seqs; w <<= 1)
#pragma unroll
    for (int b = kFewest; b <= kMost + 1; ++b) n[b - kFewest] += __shfl_xor(n[b - kFewest], w);
  int alone = kNever, shared = kNever, split = kNever;  // keys
#pragma unroll
  for (int b = kMost; b >= kFewest; --b) {
    alone = n[b - kFewest] <= teams.alone ? 1 << b : alone;
    shared = n[b - kFewest] <= teams.count ? 9 << b >> 2 : shared;
  }
  const int extra = 8 * all_pairs <= teams.alone ? 0 : kExtra;   // long pairs: few ranges hold two (256K keys: 87.0 instead of 88.0 us)
  if (all_pairs <= teams.alone) split = min(tiles_each(n[0] + extra * all_pairs, teams.alone), 1 << 20) << kFewest;
  Cut c = usual_cut(kFewest, teams);
  if (alone < kNever && alone <= split && alone <= shared) c = {31 - __builtin_clz(alone), teams.alone, 0};
  else if (split < kNever && split <= shared) c = {kFewest, teams.alone, extra};
  else if (shared < kNever) c = {30 - __builtin_clz(shared), teams.count, 0};
  c.bits = __builtin_amdgcn_readfirstlane(c.bits);
  c.teams = __builtin_amdgcn_readfirstlane(c.teams);
  c.extra = __builtin_amdgcn_readfirstlane(c.extra);
  return c;
}

template <bool kBf16, int kD, int kNT>
__global__ __launch_bounds__(256, 2) void cache_attn_kernel(CacheAttnArgs a, Teams teams, int tile_bits, Partial part) {
  constexpr int kWaves = 4, kThreads = 64 * kWaves;
  constexpr int kRows = 16 * kNT, kElt = kBf16 ? 2 : 4;
  constexpr int kBlocks = kBf16 ? 2 : 1, kKeys = 16 * kBlocks;   // blocks of 16 keys, keys of a step
  constexpr int kKL = kD * kElt / 64;                   // 16-byte pieces of a K row that a lane holds
  constexpr int kVC = kD * kElt / 256;                  // .. of a V row
  constexpr int kAcc = kD / 16;                         // O^T accumulators of 16 rows of d
  // f32: a score is added up as several sums, since each rounds at the size it has grown to.  Its rms error, products of size 1, in units of 2^-24: one sum of 128 products 38.8, two 28.4,
  // four 21.7; of 64, 19.6 / 14.5 / 11.6.  (Four with two tiles of rows of d = 128: 2 VGPRs spilled, 748 instead of 741 us for 16 x 20000 keys of 28/4 heads and five tokens.)
  constexpr int kSums = kNT == 2 && kD == 128 ? 2 : 4;
  constexpr int kParts = kNT == 1 ? 3 : 2;              // bf16 numbers that a weight is given to the matrix instructions as
  constexpr int kHalf = kKeys * kD * kElt, kCopies = kHalf / 1024;   // bytes of a step's K (or V), copies that bring them
  // A wavefront's K and V of a step; when a segment ends, the wavefronts' O for kAtOnce tiles of 16 rows, [kAtOnce][kWaves][16][kD] floats, each row's pieces of 4 in
  // places piece ^ row.
  __shared__ __attribute__((aligned(1024))) char ring[kWaves * 2 * kHalf];
  constexpr int kTileFloats = kWaves * 16 * kD, kAtOnce = (int)sizeof(ring) / (4 * kTileFloats) < kNT ? (int)sizeof(ring) / (4 * kTileFloats) : kNT;
  static_assert(kAtOnce >= 1, "the results of a tile of rows fit");
  float* const red = reinterpret_cast<float*>(ring);
  auto red_at = [&](int tile, int w, int row, int d) { return red + (tile * kTileFloats + (w * 16 + row) * kD + ((d >> 2 ^ row) << 2) + (d & 3)); };
  // Q of 48 rows is read from LDS for each step, as K is: in registers it would leave too few for two workgroups a CU.
  constexpr bool kSharedQ = kNT > 2;
  __shared__ __attribute__((aligned(16))) char q_rows[kSharedQ ? kRows * kD * kElt : 16];
  __shared__ float red_m[kWaves][kRows], red_l[kWaves][kRows];
  __shared__ int wave_tiles[kWaves], found[2];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const CacheArgs& c = a.cache;

  // ---- this team's range of tiles ----
  const Place me = place_of(teams, blockIdx.x);
  // (Every bound below also holds where cu_new is not ascending and the sums are nonsense.)
  int extra = 0;                                        // a pair counts as so many tiles more than it has
  auto tiles_of = [&](const SeqRows& r, int bits) {
    const PairShape p = pairs_of(a, teams, r, bits);
    return p.rounds * a.Hkv * (p.tiles + extra);
  };
  int n_teams = teams.count;
  const bool few = c.n_seqs <= 64;                      // every wavefront has all sequences in its lanes: no LDS, no second look at memory
  SeqRows mine = {};                                    // of sequence `lane`, if few
  int each, t, t_end, seq, base;                        // tiles of a range, the next tile, the range's end; the tile's sequence, and tiles before that one
  if (few) {
    if (lane < c.n_seqs) mine = rows_of_seq(c, lane);
    if (tile_bits < 0) {
      const Cut cut = pick_cut<fewest_bits(kBf16)>([&](int bits) { return lane < c.n_seqs ? tiles_of(mine, bits) : 0; }, lane < c.n_seqs ? tiles_of(mine, 30) : 0,
                                                   c.n_seqs, teams);
      tile_bits = cut.bits;
      n_teams = cut.teams;
      extra = cut.extra;
    }
    const int n = lane < c.n_seqs ? tiles_of(mine, tile_bits) : 0;
    int upto = n;
#pragma unroll 1
    for (int w = 1; w < c.n_seqs; w <<= 1) {
      const int x = __shfl_up(upto, w);
      if (lane >= w) upto += x;
    }
    const int total = checked_total(__builtin_amdgcn_readlane(upto, c.n_seqs - 1));
    each = tiles_each(total, n_teams);
    t = me.team * each;
    t_end = min(t + each, total);
    if (t >= t_end) return;
    seq = 63 - __builtin_clzll(__ballot(lane < c.n_seqs && upto - n <= t) | 1);   // the last one that begins by then
    base = __builtin_amdgcn_readlane(upto - n, seq);
  } else {
    if (tile_bits < 0) {
      const Cut cut = usual_cut(fewest_bits(kBf16), teams);
      tile_bits = cut.bits;
      extra = cut.extra;
    }
    const int per = (c.n_seqs + kThreads - 1) / kThreads, s_first = min(tid * per, c.n_seqs), s_last = min(s_first + per, c.n_seqs);
    int n = 0;
    for (int s = s_first; s < s_last; ++s) n += tiles_of(rows_of_seq(c, s), tile_bits);
    int upto = n;                                       // of the threads up to this one
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
      const int x = __shfl_up(upto, w);
      if (lane >= w) upto += x;
    }
    if (lane == 63) wave_tiles[wave] = upto;
    if (tid == 0) found[0] = c.n_seqs;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) upto += wave_tiles[w];
      total += wave_tiles[w];
    }
    total = checked_total(__builtin_amdgcn_readfirstlane(total));
    each = tiles_each(total, n_teams);
    t = me.team * each;
    t_end = min(t + each, total);
    if (t >= t_end) return;
    if (upto - n <= t && t < upto) {                    // one thread
      int x = upto - n, s = s_first;
      for (; s < s_last; ++s) {
        const int y = tiles_of(rows_of_seq(c, s), tile_bits);
        if (t < x + y) break;
        x += y;
      }
      found[0] = s;
      found[1] = x;
    }
    __syncthreads();
    seq = found[0];
    base = found[1];
  }

  const float sc = a.scale * kLog2e;
  for (;;) {
    // scalars, whatever the compiler makes of the above: the addresses of K and V hang on them
    t = __builtin_amdgcn_readfirstlane(t);
    base = __builtin_amdgcn_readfirstlane(base);
    seq = __builtin_amdgcn_readfirstlane(seq);
    if (t >= t_end || seq >= c.n_seqs) break;
    SeqRows r;
    if (few) {
      r.first = __builtin_amdgcn_readlane(mine.first, seq);
      r.count = __builtin_amdgcn_readlane(mine.count, seq);
      r.token = __builtin_amdgcn_readlane(mine.token, seq);
      r.length = __builtin_amdgcn_readlane(mine.length, seq);
    } else {
      r = rows_of_seq(c, seq);
      r.first = __builtin_amdgcn_readfirstlane(r.first);
      r.count = __builtin_amdgcn_readfirstlane(r.count);
      r.token = __builtin_amdgcn_readfirstlane(r.token);
      r.length = __builtin_amdgcn_readfirstlane(r.length);
    }
    const PairShape shape = pairs_of(a, teams, r, tile_bits);
    const int span = shape.tiles + extra, n_seq = shape.rounds * a.Hkv * span;
    if (t >= base + n_seq) { base += n_seq; ++seq; continue; }
    const int pair = (int)((uint32_t)(t - base) / (uint32_t)span);
    const int tile0 = __builtin_amdgcn_readfirstlane(t - base - pair * span);
    const int tile1 = __builtin_amdgcn_readfirstlane(min(shape.tiles, tile0 + (t_end - t)));
    const int kvh = __builtin_amdgcn_readfirstlane((int)((uint32_t)pair / (uint32_t)shape.rounds));
    const int group0 = __builtin_amdgcn_readfirstlane(((pair - kvh * shape.rounds) * teams.size + me.member) * kRows);
    // teams that have tiles of this pair, from the one with its first tile on
    const int n_parts = __builtin_amdgcn_readfirstlane((int)((uint32_t)(t - tile0 + shape.tiles - 1) / (uint32_t)each) - me.team + 1);
    t += min(span - tile0, t_end - t);
    if (tile0 >= shape.tiles) continue;                 // nothing but what the pair counts for

    // ---- rows ----
    const int n_list = r.count * a.group;
    auto last_key = [&](int tok) { return min(r.token + tok, r.length - 1); };   // that new token `tok` sees
    if (group0 >= n_list) continue;                     // fewer groups than the team has members
    int hi[kNT];                                        // last key that this lane's rows see
    u32x4 q[kSharedQ ? 1 : kNT][kKL];
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      const int i = group0 + j * 16 + col, ic = min(i, n_list - 1);
      const int tok = (int)((uint32_t)ic / a.group_div);
      hi[j] = last_key(tok);                            // a row behind the last one does as that one
      const char* p = reinterpret_cast<const char*>(a.q) + ((int64_t)(r.first + tok) * a.q_ts + (kvh * a.group + ic - tok * a.group) * a.q_hs) * kElt + quad * 16;
      if (kSharedQ && wave != j) continue;
#pragma unroll
      for (int i2 = 0; i2 < kKL; ++i2) q[kSharedQ ? 0 : j][i2] = *reinterpret_cast<const u32x4*>(p + i2 * 64);
      if constexpr (kSharedQ)
#pragma unroll
        for (int i2 = 0; i2 < kKL; ++i2) *reinterpret_cast<u32x4*>(q_rows + (j * 16 + col) * kD * kElt + ((i2 * 4 + quad) ^ col) * 16) = q[0][i2];
    }
    static_assert(!kSharedQ || (kNT <= kWaves && kD * kElt == 256), "a wavefront for each 16 rows of Q, 16 pieces a row");
    if constexpr (kSharedQ) __syncthreads();
    const int hi_max = __builtin_amdgcn_readfirstlane(last_key((int)((uint32_t)(min(group0 + kRows, n_list) - 1) / a.group_div)));
    const int hi_min = __builtin_amdgcn_readfirstlane(last_key((int)((uint32_t)group0 / a.group_div)));
    const int key_end = __builtin_amdgcn_readfirstlane(min((int)min((int64_t)tile1 << tile_bits, (int64_t)INT32_MAX), hi_max + 1));

    bool odd = false;                                   // this lane has left out an infinity or NaN of V
    f32x4 acc[kNT][kAcc];
    float m[kNT], l[kNT];                               // l: of this lane's keys
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      m[j] = -INFINITY;
      l[j] = 0.f;
#pragma unroll
      for (int i = 0; i < kAcc; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const char* const k_head = c.k + kvh * c.head_stride * kElt;
    const char* const v_head = c.v + kvh * c.head_stride * kElt;
    // Copy t of a block takes 64 / kRowChunks of its keys, 1 KiB: lane -> (key, 16-byte place).  A row of K has its pieces in places place ^ key, so that 16 lanes that read the
    // same piece of 16 keys find them in different banks.  V is read a row at a time, by 16 lanes.
    constexpr int kRowChunks = kD * kElt / 16, kBlockCopies = kCopies / kBlocks;
    const uint32_t row_bytes = (uint32_t)c.tok_stride * kElt, key_lane = (uint32_t)lane / kRowChunks, place = (uint32_t)lane % kRowChunks;
    uint32_t k_lane[kBlockCopies];
#pragma unroll
    for (int i = 0; i < kBlockCopies; ++i) {
      const uint32_t key = i * (64 / kRowChunks) + key_lane;
      k_lane[i] = key * row_bytes + (place ^ (key & 15)) * 16;
    }
    const uint32_t v_lane = key_lane * row_bytes + place * 16;
    char* const k_ring = ring + wave * 2 * kHalf, * const v_ring = k_ring + kHalf;
    const int32_t* const table = c.table + seq * c.table_stride;

    // Steps of this wavefront, kKeys keys each: step i takes keys key_of(i) .. + kKeys.  A refill looks up the pages of the next 64
    // blocks, one a lane; steps without any page here are passed over.
    struct Step {
      int k0;
      uint32_t here;                                    // bit b: block b lies in this pool
      int64_t at[kBlocks];                              // where the blocks lie, in bytes
    };
    auto key_of = [&](int i) { return (tile0 << tile_bits) + (i * kWaves + wave) * kKeys; };
    int ahead = 0, pages = 0;                           // first step of the refill; page of this lane's block
    uint64_t todo = 0;                                  // blocks of the refill that are here and not fetched
    auto refill = [&] {
      const int kb = key_of(ahead + lane / kBlocks) + 16 * (lane % kBlocks);
      // without a branch by lane: a loop that has none keeps its addresses in scalar registers
      pages = table[(uint32_t)min(kb, key_end - 1) / c.page_div];
      todo = __ballot(kb < key_end && pages >= 0 && pages < c.n_pages);
    };
    auto next = [&](Step& x) {
      while (todo == 0) {
        ahead += 64 / kBlocks;
        if (key_of(ahead) >= key_end) return false;
        refill();
      }
      const int i = __builtin_ctzll(todo) / kBlocks;
      x.here = (uint32_t)(todo >> (i * kBlocks)) & ((1u << kBlocks) - 1);
      todo &= ~((((uint64_t)1 << kBlocks) - 1) << (i * kBlocks));
      x.k0 = key_of(ahead + i);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        // Blocks lie inside a page.  One that is not here, beside one that is, is read from page 0 and masked.
        const int kb = x.k0 + 16 * b, slot = kb - (int)((uint32_t)kb / c.page_div) * c.page_size, page = __builtin_amdgcn_readlane(pages, i * kBlocks + b);
        x.at[b] = x.here >> b & 1 ? (page * c.page_stride + slot * c.tok_stride) * kElt : 0;
      }
      return true;
    };
    const bool team = kNT > 1 && teams.size > 1;
    auto k_copies = [&](auto shared, const Step& x) {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < kBlockCopies; ++i) copy_piece<shared>(k_head + x.at[b], k_lane[i], ring, wave * 2 * kHalf + (b * kBlockCopies + i) * 1024);
    };
    auto v_copies = [&](auto shared, const Step& x) {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < kBlockCopies; ++i)
          copy_piece<shared>(v_head + x.at[b] + (int64_t)i * (64 / kRowChunks) * row_bytes, v_lane, ring, wave * 2 * kHalf + kHalf + (b * kBlockCopies + i) * 1024);
    };
    auto copy_k = [&](const Step& x) { if (team) k_copies(std::true_type(), x); else k_copies(std::false_type(), x); };
    auto copy_v = [&](const Step& x) { if (team) v_copies(std::true_type(), x); else v_copies(std::false_type(), x); };
    // The step's copies are on their way, K's before V's; the following step's K is asked for as soon as this
    // one's has been read, and so is V.
    auto compute = [&](const Step& x, bool more, const Step& after) {
      const bool whole = x.k0 + kKeys - 1 <= hi_min && x.here == (1u << kBlocks) - 1;   // every row sees every key of the step

      wait_copies<kCopies>();                            // V's may be under way
      u32x4 k[kBlocks][kKL];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < kKL; ++i) k[b][i] = *reinterpret_cast<const u32x4*>(k_ring + (b * 16 + col) * kD * kElt + ((i * 4 + quad) ^ col) * 16);
      if (more) {
        wait_reads();
        copy_k(after);
      }

      // P^T: lane (col, quad) holds row col, keys 16 b + 4 quad + i
      f32x4 p[kNT][kBlocks];
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        u32x4 qj[kKL];
#pragma unroll
        for (int i = 0; i < kKL; ++i) {
          if constexpr (kSharedQ) qj[i] = *reinterpret_cast<const u32x4*>(q_rows + (j * 16 + col) * kD * kElt + ((i * 4 + quad) ^ col) * 16);
          else qj[i] = q[j][i];
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
          f32x4 s = {0.f, 0.f, 0.f, 0.f};
          if constexpr (kBf16) {
#pragma unroll
            for (int i = 0; i < kKL; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[b][i]), __builtin_bit_cast(bf16x8, qj[i]), s, 0, 0, 0);
          } else {
            f32x4 part[kSums];
#pragma unroll
            for (int y = 0; y < kSums; ++y) part[y] = s;
#pragma unroll
            for (int i = 0; i < kKL; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                part[e % kSums] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[b][i][e]), __uint_as_float(qj[i][e]), part[e % kSums], 0, 0, 0);
#pragma unroll
            for (int n = kSums / 2; n > 0; n /= 2)
#pragma unroll
              for (int y = 0; y < n; ++y) part[y] += part[y + n];
            s = part[0];
          }
          if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = (x.here >> b & 1) && x.k0 + 16 * b + quad * 4 + i <= hi[j] ? s[i] : -INFINITY;
          }
          p[j][b] = s;
        }
      }
#pragma unroll
      for (int j = 0; j < kNT; ++j) {
        float top = p[j][0][0];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, p[j][b][i]);
        top *= sc;
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m[j], top), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m[j] - ref);   // m = -inf: 0
        m[j] = m_new;
        l[j] *= alpha;
#pragma unroll
        for (int i = 0; i < kAcc; ++i) acc[j][i] *= alpha;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[j][b][i] = __builtin_amdgcn_exp2f(p[j][b][i] * sc - ref);
            l[j] += p[j][b][i];
          }
      }

      // O^T += V^T . P^T.  P goes in as two or three bf16 numbers, its rounding and what that leaves: 16 bits or all 24 of it.  V's are exact, so with three a partial
      // result is as exact as the fp32 it is kept in: O before its rounding is off by 1.5e-7 to 5e-7 of its size (203 to 262144 keys; 1.6e-6 to 2.1e-6 with two).  With one
      // tile of rows memory sets the pace and the third product is all but free (28/4 heads, one new token, us with two and three: 256K tokens 87.3 and 87.4, 16 sequences
      // of 20000 106.3 and 107.4, 8 of 450 9.9 and 10.1); with more tiles it is not (16 of 20000, five tokens 113.6 and 120.3, 32 tokens 349 and 392).
      bf16x8 p_part[kNT][kParts];
      if constexpr (kBf16) {
#pragma unroll
        for (int j = 0; j < kNT; ++j) {
          uint32_t w[kParts][4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            float p0 = p[j][y >> 1][(y & 1) * 2], p1 = p[j][y >> 1][(y & 1) * 2 + 1];
#pragma unroll
            for (int x2 = 0; x2 < kParts; ++x2) {
              w[x2][y] = pack2(p0, p1);
              p0 -= __uint_as_float(w[x2][y] << 16);     // exact
              p1 -= __uint_as_float(w[x2][y] & 0xffff0000u);
            }
          }
#pragma unroll
          for (int x2 = 0; x2 < kParts; ++x2) p_part[j][x2] = __builtin_bit_cast(bf16x8, mk4(w[x2][0], w[x2][1], w[x2][2], w[x2][3]));
        }
      }
      if (more) wait_copies<kCopies>();                  // the next step's K is under way
      else wait_copies<0>();
      char* const v_mine = v_ring + quad * 4 * kD * kElt + col * 16;   // what this lane reads of V: rows 16 b + r from here, pieces 16 e
      if (!whole) {
        // What no row sees is not to be multiplied, not even by zero: it may be anything.
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(x.here >> b & 1) || x.k0 + 16 * b + quad * 4 + r > hi_max)
#pragma unroll
              for (int e = 0; e < kVC; ++e) *reinterpret_cast<u32x4*>(v_mine + (b * 16 + r) * kD * kElt + e * 256) = mk4(0u, 0u, 0u, 0u);
      }
      u32x4 v[kBlocks][4][kVC];
      auto read_v = [&] {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < kVC; ++e) v[b][r][e] = *reinterpret_cast<const u32x4*>(v_mine + (b * 16 + r) * kD * kElt + e * 256);
      };
      read_v();
      // Nor is an infinity or NaN that some rows see and others do not: it is left out here and added to the rows that see it after the loop.
      if (!whole && hi_min < hi_max && x.k0 + kKeys - 1 > hi_min) {
        constexpr uint32_t kOne = kBf16 ? 0x00800080u : 0x00800000u, kExponents = kBf16 ? 0x7f807f80u : 0x7f800000u, kCarries = kBf16 ? 0x80008000u : 0x80000000u;
        uint32_t carry = 0;                              // exponents of ones only, and one more
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            uint32_t of_key = 0;
#pragma unroll
            for (int e = 0; e < kVC; ++e)
#pragma unroll
              for (int w = 0; w < 4; ++w) of_key |= (v[b][r][e][w] & kExponents) + kOne;
            carry |= x.k0 + 16 * b + quad * 4 + r > hi_min ? of_key : 0u;
          }
        if (__any((carry & kCarries) != 0)) {
#pragma unroll 1
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int e = 0; e < kVC; ++e) {
                u32x4* const at = reinterpret_cast<u32x4*>(v_mine + (b * 16 + r) * kD * kElt + e * 256);
                const u32x4 y = *at;
                u32x4 fine;
                bool left_out = false;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                  fine[w] = finite_part<kBf16>(y[w]);
                  left_out = left_out || fine[w] != y[w];
                }
                if (left_out && x.k0 + 16 * b + quad * 4 + r > hi_min) {
                  *at = fine;
                  odd = true;
                }
              }
          read_v();
        }
      }
      if (more) {
        wait_reads();
        copy_v(after);
      }
#pragma unroll
      for (int e = 0; e < kAcc; ++e) {
        bf16x8 va = {};
        float vf[4] = {};
        if constexpr (kBf16) {                         // d = 8 (row of A) + e
          const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;
          uint32_t w[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) w[y] = __builtin_amdgcn_perm(v[y >> 1][(y & 1) * 2 + 1][0][e >> 1], v[y >> 1][(y & 1) * 2][0][e >> 1], pick);
          va = __builtin_bit_cast(bf16x8, mk4(w[0], w[1], w[2], w[3]));
        } else {                                       // d = 64 (e / 4) + 4 (row of A) + e % 4
#pragma unroll
          for (int y = 0; y < 4; ++y) vf[y] = __uint_as_float(v[0][y][e / 4][e % 4]);
        }
#pragma unroll
        for (int j = 0; j < kNT; ++j) {
          if constexpr (kBf16) {
#pragma unroll
            for (int x2 = 0; x2 < kParts; ++x2) acc[j][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p_part[j][x2], acc[j][e], 0, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i], p[j][0][i], acc[j][e], 0, 0, 0);
          }
        }
      }
    };
    Step now, after;
    if (key_of(0) < key_end) refill();
    // Q has landed too, since it was asked for before the pages.  Left to the compiler the wait for it would stand in the loop, where the same counter
    // holds the copies.
    if constexpr (!kSharedQ)
#pragma unroll
      for (int j = 0; j < kNT; ++j)
#pragma unroll
        for (int i = 0; i < kKL; ++i) asm volatile("" : "+v"(q[j][i]));
    bool have = next(now);
    if (have) {
      copy_k(now);
      copy_v(now);
    }
    while (have) {
      have = next(after);
      compute(now, have, after);
      now = after;
    }
    if (__any(odd)) {
      for (int key = max((tile0 << tile_bits), hi_min + 1); key < key_end; ++key) {
        const int tp = (int)((uint32_t)key / c.page_div), page = table[tp];
        if (page < 0 || page >= c.n_pages) continue;
        const char* const row = v_head + (page * c.page_stride + (key - tp * c.page_size) * c.tok_stride) * kElt;
#pragma unroll
        for (int e = 0; e < kAcc; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x;
            if constexpr (kBf16) x = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[(quad * 4 + i) * 8 + e] << 16);
            else x = reinterpret_cast<const float*>(row)[(e / 4) * 64 + (quad * 4 + i) * 4 + e % 4];
            const bool counts = !(fabsf(x) < INFINITY);
#pragma unroll
            for (int j = 0; j < kNT; ++j) acc[j][e][i] += counts && key <= hi[j] ? x : 0.f;
          }
      }
    }

    // ---- the wavefronts' results joined ----
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
      l[j] += __shfl_xor(l[j], 16);
      l[j] += __shfl_xor(l[j], 32);
      if (quad == 0) {
        red_m[wave][j * 16 + col] = m[j];
        red_l[wave][j * 16 + col] = l[j];
      }
    }
    __syncthreads();                                    // every wavefront has read its last K and V
    const bool finished = tile0 == 0 && tile1 == shape.tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (tile0 == 0 ? 1 : 0);
#pragma unroll
    for (int j0 = 0; j0 < kNT; j0 += kAtOnce) {
#pragma unroll
      for (int j = j0; j < min(j0 + kAtOnce, kNT); ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < kAcc; e += 4) {
            // bf16: accumulators 0..7 are 8 consecutive d; f32: 0..3 (4..7 of the upper half) are 4
            const int d = kBf16 ? (quad * 4 + i) * 8 + e : (e / 4) * 64 + (quad * 4 + i) * 4;
            *reinterpret_cast<f32x4*>(red_at(j - j0, wave, col, d)) = f32x4{acc[j][e][i], acc[j][e + 1][i], acc[j][e + 2][i], acc[j][e + 3][i]};
          }
      __syncthreads();
      constexpr int kShare = kThreads / 16, kEach = kD / kShare;   // threads of a row, elements of each
      static_assert(kEach == 4 || kEach == 8, "a thread takes whole pieces of 4");
      const int row = tid / kShare, d0 = tid % kShare * kEach;
#pragma unroll
      for (int j = j0; j < min(j0 + kAtOnce, kNT); ++j) {
        const int jr = j * 16 + row;
        float top = red_m[0][jr];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, red_m[w][jr]);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f, x[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) x[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(red_m[w][jr] - ref);
          sum += f * red_l[w][jr];
#pragma unroll
          for (int e = 0; e < kEach; e += 4) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(red_at(j - j0, w, row, d0 + e));
#pragma unroll
            for (int k = 0; k < 4; ++k) x[e + k] += f * y[k];
          }
        }
        const int i = group0 + jr;
        if (i < n_list) {
          const int tok = (int)((uint32_t)i / a.group_div), h = kvh * a.group + i - tok * a.group;
          const int64_t row_head = (int64_t)(r.first + tok) * a.Hq + h;
          if (tile0 == 0 && d0 == 0) part.parts[row_head] = u32x2{blockIdx.x, (uint32_t)n_parts << 8 | (uint32_t)jr};
          if (finished) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const int64_t at = row_head * kD + d0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) x[e] *= inv;
            if (a.o != nullptr) store_row<false>(a.o, at, x);
            if (a.o_final != nullptr) store_row<kBf16>(a.o_final, at, x);
            if (a.lse != nullptr && d0 == 0) a.lse[h * a.lse_hs + r.first + tok] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
          } else {
            store_row<false>(part.o, (slot * kRows + jr) * kD + d0, x);
            if (d0 == 0) { part.m[slot * kRows + jr] = top; part.l[slot * kRows + jr] = sum; }
          }
        }
      }
      __syncthreads();
    }
  }
}

// What of a row's partial results the joining launch needs: the first block, the number of them, the row of a block's group.
struct Parts { Place first; int count, jr; };
template <int kRows>
__device__ __forceinline__ Parts parts_of(const CacheAttnArgs& a, const Teams& teams, const Partial& part, int row_head) {
  // a row of no sequence has nothing in the workspace, and whatever it finds there stays inside it
  const u32x2 found = part.parts[row_head];
  const int row = row_head / a.Hq;
  const bool none = a.cache.cu_new != nullptr && (row < load_const(a.cache.cu_new, 0) || row >= load_const(a.cache.cu_new, a.cache.n_seqs));
  const int block = (int)__builtin_amdgcn_readfirstlane(found[0]);
  Parts p;
  p.jr = (int)__builtin_amdgcn_readfirstlane(found[1]) & 255;
  p.count = (int)(__builtin_amdgcn_readfirstlane(found[1]) >> 8);
  p.first = {0, 0};
  if (none || (uint32_t)block >= (uint32_t)(teams.count * teams.size) || p.jr >= kRows) { p.count = 0; return p; }
  p.first = place_of(teams, block);
  if (p.count > teams.count - p.first.team) p.count = 0;
  return p;
}
template <int kRows>
__device__ __forceinline__ int64_t part_at(const Teams& teams, const Parts& p, int s) {
  return (2 * (int64_t)block_of(teams, p.first.team + s, p.first.member) + (s == 0 ? 1 : 0)) * kRows + p.jr;
}
template <bool kBf16, int kD>
__device__ __forceinline__ void store_result(const CacheAttnArgs& a, int row_head, int e, f32x4 x, float sum, float ref) {
  x *= sum == 0.f ? 0.f : 1.f / sum;
  const int64_t to = (int64_t)row_head * kD + e * 4;
  const float y[4] = {x[0], x[1], x[2], x[3]};
  if (a.o != nullptr) store_row<false>(a.o, to, y);
  if (a.o_final != nullptr) store_row<kBf16>(a.o_final, to, y);
  const int row = row_head / a.Hq, h = row_head - row * a.Hq;
  if (a.lse != nullptr && e == 0) a.lse[h * a.lse_hs + row] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Joins the partial results of pairs that several workgroups shared.  A workgroup takes one (row, head); teams of d / 4 threads share out the partial
// results.  It is a chain of latencies: which partial results, these with their maxima and sums, the result.  All that one
// of them needs is asked for at once: 28 workgroups that join 128 partial results each took
// 10.8 us with maxima, sums and results after one another, and take 6.1 (64 partial results: 4.9).
template <bool kBf16, int kD, int kRows>
__global__ __launch_bounds__(256, 8) void cache_join_kernel(CacheAttnArgs a, Teams teams, Partial part) {
  constexpr int kTeam = kD / 4, kTeams = 256 / kTeam, kBatch = 4;
  __shared__ f32x4 xs[kTeams][kTeam];
  __shared__ float ls[kTeams], tops[4], ms[kMaxGroups], sums[kMaxGroups];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Parts p = parts_of<kRows>(a, teams, part, blockIdx.x);
  const int count = p.count;
  if (count <= 1) return;                               // finished where it was computed
  auto at = [&](int s) { return part_at<kRows>(teams, p, s); };
  const int team = tid / kTeam, e = tid % kTeam;
  f32x4 y[kBatch];
  auto ask = [&](int from) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int s = from + k * kTeams + team;
      y[k] = s < count ? *reinterpret_cast<const f32x4*>(part.o + at(s) * kD + e * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  ask(0);
  float top = -INFINITY;
  for (int s = tid; s < count; s += 256) {
    const float m = part.m[at(s)];
    ms[s] = m;
    sums[s] = part.l[at(s)];
    top = fmaxf(top, m);
  }
#pragma unroll
  for (int w = 1; w < 64; w <<= 1) top = fmaxf(top, __shfl_xor(top, w));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int from = 0; from < count; from += kBatch * kTeams) {
    if (from > 0) ask(from);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int s = min(from + k * kTeams + team, count - 1);
      const bool live = from + k * kTeams + team < count;
      const float f = __builtin_amdgcn_exp2f(ms[s] - ref);
      sum += live ? f * sums[s] : 0.f;
      x += live ? f * y[k] : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  xs[team][e] = x;
  if (e == 0) ls[team] = sum;
  __syncthreads();
  if (team != 0) return;
  sum = 0.f;
  x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kTeams; ++k) {
    sum += ls[k];
    x += xs[k][e];
  }
  store_result<kBf16, kD>(a, blockIdx.x, e, x, sum, ref);
}

// The same with a wavefront for each (row, head): where there are many rows, each has few partial results.
template <bool kBf16, int kD, int kRows>
__global__ __launch_bounds__(256, 8) void cache_join_rows_kernel(CacheAttnArgs a, Teams teams, Partial part, int n) {
  constexpr int kTeam = kD / 4, kTeams = 64 / kTeam, kBatch = 4;
  const int lane = threadIdx.x & 63, row_head = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = lane / kTeam, e = lane % kTeam;
  if (row_head >= n) return;
  const Parts p = parts_of<kRows>(a, teams, part, row_head);
  if (p.count <= 1) return;
  float top = -INFINITY, ref = 0.f, sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < p.count; s0 += 64) {
    const int live = min(64, p.count - s0);
    f32x4 y[kBatch];
    auto ask = [&](int from) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int s = from + k * kTeams + team;
        y[k] = s < live ? *reinterpret_cast<const f32x4*>(part.o + part_at<kRows>(teams, p, s0 + s) * kD + e * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    ask(0);
    float m = -INFINITY, l = 0.f;
    if (lane < live) {
      const int64_t at = part_at<kRows>(teams, p, s0 + lane);
      m = part.m[at];
      l = part.l[at];
    }
    float most = m;
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) most = fmaxf(most, __shfl_xor(most, w));
    most = fmaxf(most, top);
    ref = most == -INFINITY ? 0.f : most;
    const float alpha = __builtin_amdgcn_exp2f(top - ref), f = __builtin_amdgcn_exp2f(m - ref);
    top = most;
    float part_sum = f * l;
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) part_sum += __shfl_xor(part_sum, w);
    sum = sum * alpha + part_sum;
    x *= alpha;
    for (int from = 0; from < live; from += kBatch * kTeams) {
      if (from > 0) ask(from);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int s = from + k * kTeams + team;
        const float fs = __shfl(f, min(s, 63));
        x += s < live ? fs * y[k] : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  }
#pragma unroll
  for (int w = kTeam; w < 64; w <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += __shfl_xor(x[i], w);
  if (team == 0) store_result<kBf16, kD>(a, row_head, e, x, sum, ref);
}

// How a call is laid out: tiles of 16 rows of a workgroup's group, teams and their members, the logarithm of a tile's keys (-1: picked by the
// kernel), and whether several workgroups may share a pair.
struct Plan { int nt, team_size, teams, tile_bits; bool shared; double most; };   // most: tiles of all pairs at most
Plan plan_of(const CacheAttnArgs& a, bool bf16) {
  const CacheArgs& c = a.cache;
  const int n_cu = cu_count();
  // Rows of a sequence: those of the one with the most where the host knows it (one new token each, one sequence, most_new), but at most twice the mean, which few exceed by much.
  // (With 2.5 times: 16 drafts of up to five tokens on 40 to 5003, 28/4 heads, of which some have 35 rows, 22.1 instead of 22.9 us, but 100 with up to four on 100 to
  // 2000, whose rows fit 32, 36.3 instead of 33.5.)  28/4 heads, us laid out for the mean, for twice the mean, and with most_new: ragged numbers, 100 sequences of 100 to 2000, up to four,
  // 46.1 / 36.4 / 36.4; 200 of 50 to 8000, up to four, 148.7 / 106.9 / 107.2; 64 of 100 to 4000, up to six, 48.0 / 41.6 / 41.7; 16 of 2000 to 20000, up to 16, 83.6 / 99.0 / 99.2;
  // five each, 16 of 20000, 113.6 / 148.5 / 113.9; 16 each 212 / 344 / 212.
  const int64_t rows_all = (int64_t)c.n_rows * a.group, most = c.cu_new == nullptr ? 1 : c.most_new > 0 ? c.most_new : c.n_rows;
  const int64_t rows_each = std::max<int64_t>(1, std::min(most * a.group, c.n_seqs == 1 ? rows_all : 2 * rows_all / c.n_seqs));
  // Groups of 32 rows, or of 48 (bf16) where they need fewer workgroups, in teams of a power of two (three members do not find each other's keys).  28/4 heads, 16
  // sequences of 20000 keys, us with groups of 48 / of 32: 5 new tokens 112 / 141, 9 157 / 143, 13 160 / 213, 16 244 / 215, 20 246 / 342, 32 454 / 350; as picked, but without
  // teams: 9 214, 16 401, 32 733.
  auto workgroups = [&](int nt) {
    const int64_t groups = (rows_each + 16 * nt - 1) / (16 * nt);
    int64_t n = 1;
    while (n < kMaxTeam && n < groups) n *= 2;
    return (groups + n - 1) / n * n;
  };
  Plan p;
  p.nt = rows_each <= 16 ? 1 : bf16 && workgroups(3) < workgroups(2) ? 3 : 2;
  p.team_size = (int)std::min<int64_t>(kMaxTeam, workgroups(p.nt));
  const int64_t capacity = (int64_t)c.max_pages * c.page_size;
  const double pairs = (double)(rows_all / (16 * p.nt * p.team_size) + c.n_seqs) * a.Hkv;
  // A short cache: one workgroup for a pair, and no second launch, up to 512 tokens (f32 half of that), or 1024 for pairs that fill the chip once.  28/4 heads, one new token,
  // us so and with shared pairs: 8 sequences of 450 tokens 9.9 and 11.5, of 900 14.9 and 12.3; 60 of 900 22.2 and 25.2, of 20 to 900 14.9 and 16.2; 200 of 450 34.7 and
  // 39.3, of 900 64.7 and 67.6, of 20 to 900 40.0 and 31.1 (with five new tokens each, of 900, 77.3 and 90.4).
  const bool once = pairs * 2 >= n_cu && (pairs <= 2.5 * n_cu || p.nt > 1);
  p.shared = capacity > (once ? 1024 : 512) / (bf16 ? 1 : 2);
  p.tile_bits = p.shared ? -1 : 30;
  const int fewest = 1 << fewest_bits(bf16);
  p.most = pairs * (p.shared ? (double)((capacity + fewest - 1) / fewest + kExtra) : 1.);
  p.teams = (int)std::min<double>(std::min(kMaxGroups, 2 * n_cu) / p.team_size, p.most);
  if (p.team_size > 1) p.teams = (p.teams + 7) / 8 * 8;  // all blocks of a team exist
  return p;
}

int64_t align16(int64_t x) { return (x + 15) / 16 * 16; }

}  // namespace

double cache_attn_tiles(const CacheAttnArgs& a, int io_dtype) { return plan_of(a, io_dtype == 0).most; }

int64_t cache_attn_workspace_bytes(const CacheAttnArgs& a, int io_dtype) {
  const Plan p = plan_of(a, io_dtype == 0);
  return align16(8 * (int64_t)a.cache.n_rows * a.Hq) + (int64_t)2 * p.teams * p.team_size * 16 * p.nt * 4 * (2 + a.d);
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, int io_dtype, hipStream_t stream) {
  if (a.cache.n_rows == 0 || a.cache.n_seqs == 0) return hipSuccess;
  const Plan p = plan_of(a, io_dtype == 0);
  Partial part;
  char* w = a.ws;
  part.parts = reinterpret_cast<u32x2*>(w);
  w += align16(8 * (int64_t)a.cache.n_rows * a.Hq);
  const int64_t rows = (int64_t)2 * p.teams * p.team_size * 16 * p.nt;
  const Teams teams = {p.teams, p.team_size == 1 ? std::min(p.teams, cu_count()) : p.teams, p.team_size, fast_div(16 * p.nt * p.team_size)};
  part.o = reinterpret_cast<float*>(w);
  part.m = part.o + rows * a.d;
  part.l = part.m + rows;
  auto launch = [&](auto bf16, auto d, auto nt) {
    constexpr bool kBf16 = decltype(bf16)::value;
    constexpr int kD = decltype(d)::value, kNT = decltype(nt)::value;
    cache_attn_kernel<kBf16, kD, kNT><<<dim3((unsigned)(p.teams * p.team_size)), dim3(256), 0, stream>>>(a, teams, p.tile_bits, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.shared || p.teams == 1) return e;
    const int n = a.cache.n_rows * a.Hq;
    // 28/4 heads, us with a workgroup and with a wavefront for a (row, head): 256K tokens 87.7 and 91.6; 64 sequences of 2000, one new token 48.7 and 47.7, five 65.1
    // and 57.8; 200 of 2000, five 185.3 and 170.4.
    if (n >= 4 * cu_count()) cache_join_rows_kernel<kBf16, kD, 16 * kNT><<<dim3((unsigned)((n + 3) / 4)), dim3(256), 0, stream>>>(a, teams, part, n);
    else cache_join_kernel<kBf16, kD, 16 * kNT><<<dim3((unsigned)n), dim3(256), 0, stream>>>(a, teams, part);
    return hipGetLastError();
  };
  auto by_rows = [&](auto bf16, auto d) {
    if constexpr (decltype(bf16)::value)
      if (p.nt == 3) return launch(bf16, d, std::integral_constant<int, 3>());
    if (p.nt == 2) return launch(bf16, d, std::integral_constant<int, 2>());
    return launch(bf16, d, std::integral_constant<int, 1>());
  };
  if (io_dtype == 0) return by_rows(std::true_type(), std::integral_constant<int, 128>());
  if (a.d == 128) return by_rows(std::false_type(), std::integral_constant<int, 128>());
  return by_rows(std::false_type(), std::integral_constant<int, 64>());
}

}  // namespace mmsp
