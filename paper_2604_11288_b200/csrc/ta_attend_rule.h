// How a call of the attention of new tokens (ta_attend.cu) is cut, and the scratch that it takes. Host code only, but for the constants.
#pragma once

#include <stddef.h>

#ifdef __CUDACC__
#define TA_ATTEND_RULE __host__ __device__
#else
#define TA_ATTEND_RULE
#endif

constexpr int kAttendTickets = 16384;  // units and row blocks of a call whose cache rows are cut into pieces
constexpr int kAttendJoined = 4096;    // pieces of a row block, times its rows: what the last block joins in shared memory
constexpr int kAttendPieceUnit = 128;  // cache rows: whole rounds of every variant's four warps
TA_ATTEND_RULE constexpr int ta_attend_rows(int mb) { return mb == 0 ? 8 : 16 * mb; }            // query rows of a block
constexpr int ta_attend_mb(int rows) { return rows <= 8 ? 0 : rows <= 16 ? 1 : 2; }              // for so many of a unit
constexpr long long ta_attend_resident(int mb) { return 148 * (mb < 2 ? 3 : 2); }                // blocks on the device at once

// How a call is cut: query rows and warps of a block, and pieces of the cache rows. Sized for the 148 SMs of a B200 at three blocks
// each, two with 32 query rows.
struct ta_attend_plan {
  int mb, warps, row_blocks, piece, pieces, target;
};
// The smallest number of pieces that fills whole rounds of resident blocks: a last round with few blocks costs as much as a full
// one. bf16 is bound by memory and content with 85 % of a round, the 8-bit formats by instructions (95 %). us at 1, 2, 3, 4, 6, 8
// pieces: 128 units of 32768 bf16 rows 563, 333, 441, 343, 349, 354; 288 units of 16384 e4m3 rows -, 312, 252, 257, 265, -.
// Where every sequence has a length of its own, and all units fit at once, the pieces are cut on the device from the sum of the
// lengths, with room for twice as many: 4 x 4 units of 100001 to 131072 int8 rows 154 us, 168 with pieces of max_len / 27 (127 by now); not with
// more units (512 units of 2048 to 16384 e4m3 rows 308 and 294), whose empty blocks cost more than evenness brings.
// Many short units: blocks of two warps, twice as many an SM, whose starts and ends weigh half as much (4096 units in a step, us with
// four and two warps: 17 rows 54 and 40, 65 rows 74 and 59, 257 rows 128 and 122, 4097 rows 1418 and 1403; one warp 36, 53, 121); only up to
// 512 rows where lengths differ, which longer blocks even out less (4096 units, longest eight times the shortest, four and two warps: 256
// rows e4m3 90 and 85, bf16 86 and 75; 512 rows 117.0 and 116.0, 118 and 112; 768 rows 142.1 and 142.5, 155.8 and 156.2; 1024 rows 172 and
// 177, 208 and 213).
// With more units than fit at once lengths may differ: four rounds at least (512 units of 2048 to 16384 e4m3 rows
// -, 331, 312, 293, 294, -; 296 units of 32768 bf16 rows alike lose 1.5 %, 726 to 737).
inline ta_attend_plan ta_attend_plan_of(long long units, int rows, int max_len, bool codes, int ragged_batch) {
  ta_attend_plan p;
  p.mb = ta_attend_mb(rows);
  p.row_blocks = (rows + ta_attend_rows(p.mb) - 1) / ta_attend_rows(p.mb);
  const long long groups = units * p.row_blocks, slots = ta_attend_resident(p.mb);
  int most = groups > kAttendTickets || max_len <= kAttendPieceUnit ? 1 : (max_len + kAttendPieceUnit - 1) / kAttendPieceUnit;
  if (most > kAttendJoined / ta_attend_rows(p.mb)) most = kAttendJoined / ta_attend_rows(p.mb);
  int k = 1;
  for (; k < most; ++k) {
    const long long blocks = groups * k, rounds = (blocks + slots - 1) / slots;
    if (groups > slots && rounds < 4 && k < 4) continue;
    if (blocks * 100 >= rounds * slots * (codes ? 95 : 85)) break;
    if (rounds > 8) break;
  }
  p.piece = ((max_len + k - 1) / k + kAttendPieceUnit - 1) / kAttendPieceUnit * kAttendPieceUnit;
  if (p.piece < kAttendPieceUnit) p.piece = kAttendPieceUnit;
  p.pieces = max_len > p.piece ? (max_len + p.piece - 1) / p.piece : 1;
  p.target = 0;
  p.warps = p.mb == 0 && p.pieces == 1 && groups >= 4 * slots && (ragged_batch == 0 || max_len <= 512) ? 2 : 4;
  if (p.pieces > 1 && ragged_batch > 1 && groups <= slots) {  // (every block adds up the lengths of as many sequences)
    p.target = (int)(groups * p.pieces);
    p.pieces = 2 * p.pieces < most ? 2 * p.pieces : most;
  }
  return p;
}

// Places for the results of pieces: one for every row of every block of a call whose units are cut.
inline size_t ta_attend_slots(const ta_attend_plan& p, long long units) {
  return p.pieces > 1 ? (size_t)units * p.row_blocks * p.pieces * ta_attend_rows(p.mb) : 0;
}
// As many as a call can need that is no larger than this one: in layers, sequences and KV heads (units), query heads of a KV head and
// tokens (rows), and max_len. A smaller call may be cut into more blocks than a larger one, whose units fill the device as they are. The
// number of pieces is raised while the blocks of one less are at most eight rounds: 9 rounds where all units fit at once, twice
// that where the device cuts them, 16 otherwise; and no more than there are pieces.
inline size_t ta_attend_most_slots(long long units, int rows, int max_len) {
  size_t most = 0;
  for (int mb = 0; mb <= ta_attend_mb(rows); ++mb) {
    const int R = ta_attend_rows(mb);
    const long long groups = units * (mb < 2 ? 1 : (rows + R - 1) / R);
    long long pieces = (max_len + kAttendPieceUnit - 1) / kAttendPieceUnit;
    if (pieces > kAttendJoined / R) pieces = kAttendJoined / R;
    if (pieces < 2) continue;
    const long long rounds = 18 * ta_attend_resident(mb), blocks = groups * pieces < rounds ? groups * pieces : rounds;
    if (most < (size_t)blocks * R) most = (size_t)blocks * R;
  }
  return most;
}

struct ta_attend_sizes {  // bytes
  size_t part, part_ml;   // results of pieces, and their maxima and sums
  size_t score, row_ml;   // for the attention mass
  size_t all() const { return part + part_ml + score + row_ml; }
};
inline long long ta_attend_score_stride(int max_len) { return (max_len + 31) / 32 * 32; }
inline ta_attend_sizes ta_attend_sizes_of(long long units, int rows, int d, int max_len, size_t slots, bool with_mass) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  ta_attend_sizes z = {up(slots * d * 4), up(slots * 8), 0, 0};
  if (with_mass) {
    z.score = up((size_t)units * rows * ta_attend_score_stride(max_len) * 4);
    z.row_ml = up((size_t)units * rows * 8);
  }
  return z;
}
