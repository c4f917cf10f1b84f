// The 4-bit key/value cache: its layout, shared by the host code and the
// kernels, and the interface between them.
#ifndef FABFT_CACHE_H
#define FABFT_CACHE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fabft {

// The cache of one head is a row of tiles of 64 slots (keys). A tile holds, one
// part after the other:
//   K codes    64 rows of d/2 bytes; channel 2j in the low half of byte j
//   K scales   one byte e per slot and block of 32 channels (value 2^(e - 127),
//              255: the block is NaN), at kscale_at: the lanes that hold the rows
//              of an MFMA operand find the scales of their four 16-key blocks in
//              one 32-bit word
//   V codes    as K's
//   V scales   64 bf16
//   V sums     2 x 64 bf16: hi, then lo; hi + lo is the sum of the row's codes
//              (before the scale), exactly: hi a multiple of 16, lo of 1/2 below 16
//   V weighted sums  the same of the sum with signs (-1)^j
// One tile after the other in memory, so that a step of the attention reads
// one contiguous piece.
constexpr int kCacheTile = 64;

struct CacheTile {
  int d;
  constexpr explicit CacheTile(int d_) : d(d_) {}
  constexpr int row() const { return d / 2; }
  constexpr int blocks() const { return d / 32; }
  constexpr int kscale() const { return kCacheTile * row(); }
  constexpr int vcode() const { return kscale() + kCacheTile * blocks(); }
  constexpr int vscale() const { return vcode() + kCacheTile * row(); }
  constexpr int vsum() const { return vscale() + 2 * kCacheTile; }
  constexpr int vwsum() const { return vsum() + 4 * kCacheTile; }
  constexpr int bytes() const { return vwsum() + 4 * kCacheTile; }
  // MFMA row m of 16-key block kb of a tile is the key 16 (m >> 2) + 4 kb + (m & 3):
  // then the lane that holds the scores of rows 4g .. 4g + 3 of all four blocks holds
  // the keys 16g .. 16g + 15, those whose V the transposed read gives it
  constexpr int kscale_at(int key, int block) const {
    const int m = ((key >> 4) << 2) | (key & 3), kb = (key >> 2) & 3;
    return kscale() + (m * blocks() + block) * 4 + kb;
  }
};

struct CacheParams {
  uint8_t* cache;
  const uint16_t* q;
  uint16_t* o;
  float* resid;
  uint8_t* flags;
  const int* lengths;   // [B] keys per sequence
  const int* counts;    // [B] query rows (new tokens) per sequence, or null: all
  float* weight;        // [B, H, tiles * 64], or null
  float* stats;         // per query row 4 floats: m (exp2 domain), 1 / l (0: the row
                        // adds nothing), its last visible key, unused; null without weight
  float* ws;            // split records: m, l, c, c_w, o[d]
  unsigned long long* tickets;   // per head, row tile and split: the nonce, once it is done
  unsigned long long nonce;      // of this launch, not 0
  int B, H;             // H: key/value heads
  int tiles;            // capacity in tiles
  int Lq, R;            // query rows per query head, per key/value head
  int causal, nsplit, n_rt;
  int by_length;        // workgroups take the longest sequences first
  int wcheck;
  float sl2, decay, tau_rel, tau_abs;
};

struct CacheRows {   // append, read
  uint8_t* cache;
  uint16_t* k;
  uint16_t* v;
  long long kb, kh, kn, vb, vh, vn;   // strides in elements
  const int* start;
  const int* counts;
  int B, H, tiles, n;
};

struct CacheEvict {
  uint8_t* cache;
  uint8_t* into;        // == cache: in place
  float* weight;        // [B, H, tiles * 64]
  float* into_weight;   // [B, H, into_tiles * 64]
  const int* lengths;
  int* new_lengths;     // [B]
  int* index;           // [B, H, keep]
  int B, H, tiles, into_tiles, keep, recent;
};

// Query rows of a workgroup of the attention, for R rows per key/value head.
inline int cache_row_tile(int R) { return R <= 1 ? 1 : R <= 4 ? 4 : R <= 8 ? 8 : R <= 16 ? 16 : 32; }
// As many tiles stay with one workgroup: a merge costs 2.2 us, a round of tiles 0.9.
constexpr int kCacheFewTiles = 12;
// Splits of the keys of a cache of `tiles` tiles, a tile for each wave or more: so many that the
// workgroups fill the chip once, and no round of a few is left over. Up to 16 rows: two
// workgroups per CU (512) while each has 16 tiles or more, else one. Measured (us, splits
// at 512 and at 256 workgroups): 128 heads of 512 tiles 109 113, 64 of 512 30.0 33.4, 128 of 128
// 30.8 32.0; 32 heads of 65 tiles 13.1 11.8, 64 of 32 13.1 12.7, 8 heads of 512 21.6 18.4. Rounded
// down and up: 96 heads of 512 tiles 75.0 91.2, 132 of 256 56.8 80.3, 192 of 128 46.2 52.9, 288
// of 64 36.7 44.3.
// More rows: no more than one per CU, since the records are more too. (256 row tiles of 128
// channels: 64 tiles of keys 34.9 in one split, 51.8 in two, 256 tiles 104 and 114, 512 tiles 177
// and 177; 192 row tiles of 64 channels, 64 tiles, 27.9, 40.9 and 46.2 in three; 64 row tiles,
// 128 tiles, 28.7 in four splits, 29.7 in eight.) Between 129 and 255 row tiles that is one split,
// which leaves CUs without work; two, of 258 to 510 workgroups, are slower all the same up to 256
// tiles of keys (d = 128, one and two splits: 130 row tiles 30.8 42.2 at 64 tiles, 48.9 58.6 at 128,
// 85.5 91.2 at 256; 200 row tiles 31.1 47.3, 49.9 63.8, 85.9 96.3; d = 64, 256 tiles: 71.3 72.8 and
// 70.9 78.2) and at 512 tiles between 8% faster and 10% slower (130 row tiles: d = 64 130 120, 128
// 159 156; 200: 129 125, 159 161; 160: d = 96 146 141, 256 260 286). What rounding down costs: 128
// row tiles of 512 tiles of keys take 75.3 (d = 64) and 97.5 (128) in the two splits chosen, 70.6 and
// 92.5 in four; of 128 tiles 34.8 and 34.9, 40.3 and 40.5.
inline int cache_splits(int B, int H, int R, int tiles) {
  if (tiles <= kCacheFewTiles) return 1;
  const long long units = (long long)B * H * ((R + cache_row_tile(R) - 1) / cache_row_tile(R));
  long long ns = (R > 16 ? 256 : 512) / units;
  if (R <= 16 && tiles < 16 * ns) ns = 256 / units;
  if (ns > (tiles + 3) / 4) ns = (tiles + 3) / 4;
  return ns > 64 ? 64 : ns < 1 ? 1 : (int)ns;
}
inline int cache_record_floats(int d) { return d + 4; }

// 0, -1 (the launch failed) or kCacheGrid: the call is more than a grid holds, and nothing ran.
constexpr int kCacheGrid = -2;
// Rows n of an append or a read, and query rows B * H * G * Lq: then no 32-bit index of a row,
// or of the first row of a tile behind the last, overflows.
constexpr int kCacheMostRows = 1 << 30;

int launch_cache_append(const CacheRows& p, int d, hipStream_t s);
int launch_cache_read(const CacheRows& p, int d, hipStream_t s);
int launch_cache_attn(const CacheParams& p, int d, hipStream_t s);
int launch_cache_evict(const CacheEvict& p, int d, hipStream_t s);

}  // namespace fabft

#endif
