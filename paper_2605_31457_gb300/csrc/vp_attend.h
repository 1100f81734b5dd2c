// Definitions of vp_attend_new and vp_evict shared by the host side
// (vp_cache_api.cu) and the kernels (vp_attend.cu, vp_evict.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "vp_internal.h"

namespace vp {

// Rows of query heads (vp_rows), strides in elements.
struct RowView {
  void* data;
  int64_t sb, sn, sh;
};
// One float per cached token and kv-head (vp_weights).
struct WeightView {
  float* data;
  int64_t sb, sh;
};

constexpr int kNewWeightRows = 128;  // n_new * G of a call that accumulates weights
constexpr int kAnyTile = 32;         // cached tokens per tile of k_att_any
constexpr int kAnyRows = 16;         // most query rows per CTA of k_att_any

constexpr int kTcTile = 128;         // cached tokens per tile of k_att_tc; query rows per accumulator

// Of the workspaces, per SM: partial rows and tickets.
constexpr int kPartRows = 4 * kTcTile, kTickets = 4;

// The workspace of vp_attend_new (vp_reserve_new), offsets in bytes.
struct NewLayout {
  int max_new = 0, max_weight_new = 0;
  int z_row = 0;              // floats per row of logits
  size_t o_tk = 0, o_lse = 0, o_st = 0, o_o = 0, o_z = 0, total = 0;
};

// Which kernel serves a call (plan_attend).  `block` query rows of one
// (sequence, kv-head) are an item of the tensor-core kernels:
//   ATT_DEC  k_att_dec: at most 64 query rows, all of them one item;
//   ATT_TC1  k_att_tc: 65 to 128, one item whose tiles alternate between its
//            two softmax groups;
//   ATT_TC2  k_att_tc: 256 rows at a time, 128 for each group.
enum { ATT_ANY = 0, ATT_DEC = 1, ATT_TC1 = 2, ATT_TC2 = 3 };
constexpr int kDecRows = 64;

// Query row r of a kv-head = new token r / G, query head g * G + r % G.
struct AttendParams {
  CUtensorMap tmk, tmv;       // k_att_tc: the caches in boxes of up to 128 rows
  int tpos, gpos, bpos;       // descriptor dimensions of the token, kv-head and sequence / page axes
  int kind;                   // ATT_*
  int block, nqt;             // tensor-core kernels: query rows of an item, items per (sequence, kv-head)
  int fixed;                  // the fixed part of an item's cost, in units
  int dtype, B, H, Hkv, G, D, max_seq;
  int paged, page_size, page_shift;
  int n_new, R;               // R = n_new * G query rows per (sequence, kv-head), below 2^28
  uint32_t g_mul;             // floor(2^32 / G) + 1: row / G is its high product with the row; 0: G = 1
  RowView q, out;
  KvView k, v;
  const int32_t* seq_len;
  const int32_t* new_len;     // or NULL
  int window, sinks;
  float c_log2;               // logit scale * log2(e)
  float* lse;                 // [B][n_new][H] or NULL
  int weigh;                  // weights asked for
  WeightView w_in, w_out;     // w_in.data may be NULL
  // workspace
  unsigned* tickets;          // [kTickets * num_sms] records written of the items cut between CTAs; 0 between calls:
                              // a CTA's (two of them per SM, k_att4: three) or one for each 16 or 128 of its rows,
                              // or k_att_any's for its row blocks, which it splits where there are at most four per SM
  float* lse2;                // [B * Hkv][R] log-sum-exp in log2 units (+inf: an empty row), when weigh
  float* part_o;              // partial outputs, unnormalised
  float* part_st;             // their {maximum in log2 units, sum}
  float* z;                   // [B * Hkv][R][z_row] logits in log2 units, of visible tokens, when weigh
  int z_row;
  unsigned* err;
  int ns;                     // splits of k_att_any
  int grid;                   // CTAs of the tensor-core kernels
  int num_sms;
};

// The cached tokens that query rows with positions in [t0, t1] (t0 <= t1) see
// between them: [0, s_end) and [lo, hi), s_end <= lo when both are non-empty
// and apart; with window < 0 everything is in [lo, hi).
struct SeenRange {
  int s_end, lo, hi;
};
__host__ __device__ inline SeenRange seen_range(int t0, int t1, int window, int sinks) {
  SeenRange r;
  r.hi = t1 + 1;
  if (window < 0) {
    r.s_end = r.lo = 0;
    return r;
  }
  r.lo = window > t0 ? 0 : t0 - window + 1;
  if (window == 0) r.lo = r.hi;  // only the sinks
  r.s_end = sinks < r.hi ? sinks : r.hi;
  if (r.s_end >= r.lo) {         // one run
    r.lo = 0;
    r.s_end = 0;
    if (window == 0) r.hi = sinks < r.hi ? sinks : r.hi;
  }
  return r;
}
// The same as a list of tiles of `rows` tokens: entry u is tile u for
// u < na, else tile b0 + u - na; n entries, no tile twice.
struct TileList {
  int na, b0, n;
  __host__ __device__ int tile(int u) const { return u < na ? u : b0 + u - na; }
};
__host__ __device__ inline TileList tile_list(const SeenRange& r, int rows) {
  TileList l;
  l.na = (r.s_end + rows - 1) / rows;
  l.b0 = r.lo / rows;
  const int b1 = (r.hi + rows - 1) / rows;
  if (l.b0 < l.na) l.b0 = l.na;  // the two runs meet in one tile
  l.n = l.na + (b1 > l.b0 && r.hi > r.lo ? b1 - l.b0 : 0);
  return l;
}
__host__ __device__ inline bool sees(int j, int t, int window, int sinks) {
  return j <= t && (window < 0 || j > t - window || j < sinks);
}

// ---- The work of the tensor-core kernels.  The cost of an item is its tiles'
// plus a fixed part for loading its queries and writing its result, in thirds of
// a tile: measured, a tile takes 1.5 times as long as it would with P in one bf16
// term, and an item's fixed part as long as one (k_att_dec) or two (k_att_tc) of
// those.
// Items follow one another kv-head by kv-head, sequence by sequence, and the
// line of their costs is cut into equal parts, one per CTA: a CTA owns tiles,
// not items, so ragged lengths leave no CTA idle.  An item whose tiles lie with
// several CTAs leaves a record (m, l, O) per CTA (and group); the last CTA to
// finish joins them.
constexpr int kTileUnits = 2, kSplitUnits = 3;

struct AttItem {
  int row0, rows;  // query rows [row0, row0 + rows)
  SeenRange sr;
  TileList tl;
  __host__ __device__ int unit() const { return kSplitUnits; }
  __host__ __device__ int cost(int fixed) const { return fixed + tl.n * unit(); }
  // Tiles that start in front of position x of the item.
  __host__ __device__ int tiles_before(int x, int fixed) const {
    const int u = (x - fixed + unit() - 1) / unit();
    return x <= fixed ? 0 : u < tl.n ? u : tl.n;
  }
};
// row / G; on the device by AttendParams::g_mul.
__host__ __device__ inline int token_of_row(int row, int G, uint32_t g_mul) {
#ifdef __CUDA_ARCH__
  return g_mul ? (int)__umulhi((unsigned)row, g_mul) : row;
#else
  (void)g_mul;
  return row / G;
#endif
}
__host__ __device__ inline AttItem att_item(int len, int n, int G, int block, int qt, int window, int sinks,
                                            uint32_t g_mul = 0) {
  AttItem it;
  it.row0 = qt * block;
  const int left = n * G - it.row0;
  it.rows = left < 0 ? 0 : left < block ? left : block;
  it.sr = SeenRange{0, 0, 0};
  if (it.rows > 0) {
    const int first = len - n;
    it.sr = seen_range(first + token_of_row(it.row0, G, g_mul), first + token_of_row(it.row0 + it.rows - 1, G, g_mul),
                       window, sinks);
  }
  it.tl = tile_list(it.sr, kTcTile);
  return it;
}
// A line of `total` positions cut for at most `ctas` CTAs: CTA c owns
// [start(c), start(c + 1)); the first `extra` of them own one position more.  A
// CTA does the tiles that start in its part.  Parts are longer than a tile, so
// every CTA between those of an item's first and last tile has one of them.
struct LineCut {
  int nc, per, extra;
  __host__ __device__ LineCut() {}
  __host__ __device__ LineCut(int total, int ctas) {
    const int most = total > kSplitUnits ? total / kSplitUnits : 1;
    nc = most < ctas ? most : ctas;
    per = total / nc;
    extra = total - per * nc;
  }
  __host__ __device__ int start(int c) const { return c * per + (c < extra ? c : extra); }
  __host__ __device__ int owner(int x) const {
    const int big = extra * (per + 1);
    return x < big ? (int)((unsigned)x / (unsigned)(per + 1)) : extra + (int)((unsigned)(x - big) / (unsigned)per);
  }
};
// Few items (at most a quarter as many as CTAs) are not cut as one line: each
// gets CTAs of its own, share_count of them, so that no CTA does the end of one
// item and then the beginning of another while the rest wait (one sequence of
// 3857 tokens, 28/4 heads: 17.1 -> 15.4 us a call when it was made; with up to
// half as many items as CTAs, 32 sequences of 2816 to 6400 tokens went from 66 to
// 73 us).  Share k of m is [cost * k / m, cost * (k + 1) / m): at least half of
// `per` >= min_share(fixed), which covers the fixed part and a tile, so every share
// has a tile.
__host__ __device__ inline int min_share(int fixed) { return 2 * (fixed > kSplitUnits ? fixed + 1 : kSplitUnits); }
__host__ __device__ inline int share_count(int cost, int per) { return (cost + per - 1) / per; }

// Records and tickets of the tensor-core kernels.  Of the items whose tiles lie
// with several CTAs a CTA does at most two: the one it goes on with (c0 < cta) and
// the one it begins (c0 == cta).  Each has a record of its own there, and the CTA
// it begins at has its ticket, so none of those is used twice in a call.  An item
// whose tiles are one CTA's alone may be any of many: it must use no ticket, and
// what it writes to a record is read before the CTA's next item.
__host__ __device__ inline int record_of(int cta, int c0) { return 2 * cta + (cta == c0 ? 1 : 0); }
__host__ __device__ inline bool by_ticket(int parts) { return parts > 1; }

// The longest line a call can have (it is kept below 2^31).
inline int64_t line_bound(int64_t items, int max_seq, int fixed) {
  return items * (fixed + (int64_t)kSplitUnits * ((max_seq + kTcTile - 1) / kTcTile + 1));
}

// Splits of k_att_any: those with the least tiles on the longest way through
// the SMs, a wave being the CTAs that run at once and a CTA's start and end
// about as long as kAnyFixed tiles; at most 8 CTAs per SM, at least a tile each.
constexpr int kAnyFixed = 4;
inline int any_splits(int B, int Hkv, int R, int rows, int n_new, int window, int sinks, int max_seq, int num_sms) {
  const int64_t units = (int64_t)B * Hkv * ((R + rows - 1) / rows);
  int64_t span = max_seq;
  if (window >= 0 && (int64_t)window + n_new + sinks + 2 * kAnyTile < span)
    span = (int64_t)window + n_new + sinks + 2 * kAnyTile;
  const int64_t tiles = (span + kAnyTile - 1) / kAnyTile, wave = (int64_t)(rows <= 8 ? 3 : 2) * num_sms;
  int64_t best = 1, least = INT64_MAX;
  for (int64_t ns = 1; ns == 1 || (ns <= tiles && units * ns <= 8 * num_sms); ++ns) {
    const int64_t way = (units * ns + wave - 1) / wave * ((tiles + ns - 1) / ns + kAnyFixed);
    if (way < least) { least = way; best = ns; }
  }
  return (int)best;
}
inline int any_rows(int R) { return R <= 4 ? 4 : R <= 8 ? 8 : kAnyRows; }

inline NewLayout new_layout(int max_batch, int H, int Hkv, int D, int max_seq, int max_new, int max_weight_new,
                            int num_sms) {
  NewLayout w;
  w.max_new = max_new;
  w.max_weight_new = max_weight_new;
  const size_t G = (size_t)(H / Hkv);
  // Partial rows.  The tensor-core kernels leave up to two records per CTA (the
  // item it goes on with and the one it begins), of 16 rows at two CTAs per SM, of
  // 64 or of 256 at one, k_att4 of 8 rows at three CTAs per SM or of up to 32 at
  // two; k_att_any, whose CTAs number at most 8 per SM where it splits
  // (any_splits), one of up to kAnyRows rows each.
  const size_t rows = (size_t)kPartRows * num_sms;
  static_assert(8 * kAnyRows <= kPartRows, "k_att_any's partial rows fit");
  size_t off = 0;
  w.o_tk = off; off = ws_round(off + (size_t)kTickets * num_sms * 4);
  w.o_lse = off; off = ws_round(off + (size_t)max_batch * Hkv * max_weight_new * G * 4);
  w.o_st = off; off = ws_round(off + rows * 2 * 4);
  w.o_o = off; off = ws_round(off + rows * D * 4);
  w.z_row = (max_seq + 127) / 128 * 128;
  w.o_z = off; off = ws_round(off + (size_t)max_batch * Hkv * max_weight_new * G * w.z_row * 4);
  w.total = off;
  return w;
}

// Eviction (vp_evict).
struct EvictParams {
  int esz, B, Hkv, D, max_seq;
  int page_size, page_shift;  // of whichever cache is paged
  KvView ks, vs, kd, vd;
  int in_place;
  const int32_t* seq_len;
  int keep, sinks, recent, granularity;
  WeightView w, wd;           // wd.data may be NULL
  int32_t* kept_idx;
  int kept_cap;
  int32_t* new_len;
  unsigned* err;
  int num_sms;
};

cudaError_t configure_attend();
// Chooses the kernel (p.kind) and its launch shape; encodes the tensor maps.
void plan_attend(AttendParams& p);
cudaError_t configure_dec();
cudaError_t configure_tc();
cudaError_t launch_dec(const AttendParams& p, cudaStream_t s);
cudaError_t launch_tc(const AttendParams& p, cudaStream_t s);
cudaError_t launch_attend(const AttendParams& p, cudaStream_t s);
cudaError_t configure_evict();
cudaError_t launch_evict(const EvictParams& p, cudaStream_t s);

}  // namespace vp
