// Host rules for the tile form of a product, from its sizes alone.
#pragma once

namespace ec {

// fp32 products.  128 x 128 tiles from one per CU on (16 experts x 512 rows, d 1024, h 512 in
// 64 x 64 tiles, whose waves read a third more LDS per MFMA and meet at twice as many
// barriers: 1037 against 795 us a training step); below that 64 x 64 tiles keep more CUs busy.
constexpr long F32_BIG_TILES = 256;
// Packed rows: 64 x 128 tiles of four waves, three workgroups a CU, which end their rounds
// more evenly (us, 128 x 128 against 64 x 128: W1/W3 of 16 experts x 250 rows, d 1024, h 512
// 151 and 117, x 2000 655 and 587; dA 94 and 90, 421 and 354; 64 experts x 300 rows 316 and
// 258; dX 152 and 128, 632 and 630).  The weight gradients take them while they are at most
// one round, 768 (us, 128 x 128 against 64 x 128: dW2 of 17 x 900 rows, d 512, h 512, 544
// tiles of 64 x 128, 139 and 119; 24 x 250, d 512, h 512, 768 tiles, 51 and 44; 20 x 400, d
// 640, h 512, 800 tiles, 74 and 80; 31 x 258, d 512, h 512, 992 tiles, 54 and 66; 16 x 250, d
// 1024, h 512, 1024 tiles, 53 and 59).  64 x 64 tiles are level or slower for them (8 x 250, d
// 512, h 256, dW1/dW3 26 and 19, dW2 17.0 and 17.7; 3 x 600, d 256, h 256 30.3 and 31.0).
constexpr long F32_WIDE_ROUND = 768;

enum class F32Form { SMALL /* 64 x 64 */, WIDE /* 64 x 128 */, BIG /* 128 x 128 */ };

// Who has the rows: every batch M of its own, or packed batches, whose rows are the product's
// or (weight gradients) its contraction's.
enum class F32Rows { UNIFORM, PACKED, PACKED_K };

// `batches` outputs of M rows and `width` columns (W1/W3: those of both).
inline F32Form f32_form(F32Rows rows, int batches, int M, int width) {
  if (rows == F32Rows::PACKED) return F32Form::WIDE;
  const long big = (long)batches * ((M + 127) / 128) * ((width + 127) / 128);
  const long wide = (long)batches * ((M + 63) / 64) * ((width + 127) / 128);
  if (rows == F32Rows::PACKED_K) return wide <= F32_WIDE_ROUND ? F32Form::WIDE : F32Form::BIG;
  return big < F32_BIG_TILES ? F32Form::SMALL : F32Form::BIG;
}

// ---- bf16 products over packed rows or over all tokens -------------------------------

// The rows of a product: packed batches, whose counts the host does not know, of max_rows
// in all, or (the shared experts) one batch of max_rows.
struct RowsOf {
  bool packed;
  int batches;
  long max_rows;
};

// Rounds of tiles of bm rows, nt to a row block, on the chip: how many a CU takes one after
// the other (`at_once` run together); past the first, half a tile is the expected wait for
// the last.  Packed batches are expected to take half a row block more each than max_rows
// fills, one at least.
inline double tile_rounds(const RowsOf& r, int bm, int nt, int at_once) {
  double blocks = (double)((r.max_rows + bm - 1) / bm);
  if (r.packed) {
    blocks = (double)r.max_rows / bm + 0.5 * r.batches;
    if (blocks < r.batches) blocks = r.batches;
  }
  const double t = blocks * nt / at_once;
  return t <= 1.0 ? 1.0 : t + 0.5;
}

// Few rows an expert in enough tiles only stream the weights: 256-row tiles, whose short
// last blocks are then all there is.
inline bool rows_stream(const RowsOf& r, int nt) {
  return r.max_rows <= 96l * r.batches && (long)r.batches * nt > 128;
}

enum class FwdForm { ROWS_256, ROWS_192, ROWS_128, SQUARE_128 };

// Forward products: 256-row tiles, or smaller ones where those leave CUs idle or end in a
// poorly filled round, by tile_rounds and the time of a tile relative to a 256 x 256 one (192
// rows 0.85; 128 rows, three stages, 0.65; 128 x 128 0.4).  Measured with rows spread by a
// factor of 1.35, us of W1/W3 in tiles of 256, 192, 128 rows and 128 x 128: 8 experts x 128
// rows, d 2048, h 1024 54, 46, 38 and 31; x 600 65, 52, 65 and 77; 16 x 300, d 1024, h 512
// 38, 28, 23 and 32; 64 x 128, d 2048, h 1024 186, 183, 164 and 197; x 256 193, 222, 208 and
// 284; x 512 296, 362, 372 and 503; 64 rows (streaming) 144, 143, 159 and 157.  W2 follows
// (8 x 128 31, 24, 20, 17; 64 x 128 114, 112, 95, 105; x 512 180, 206, 197, 267).
inline FwdForm fwd_rows_form(const RowsOf& r, int width) {
  const int nt = (width + 255) / 256, nt128 = (width + 127) / 128;
  if (rows_stream(r, nt)) return FwdForm::ROWS_256;
  const double t256 = tile_rounds(r, 256, nt, 256), t192 = 0.85 * tile_rounds(r, 192, nt, 256);
  const double t128 = 0.65 * tile_rounds(r, 128, nt, 256);
  const double tsq = 0.4 * tile_rounds(r, 128, nt128, 256);
  if (tsq < t128 && tsq < t192 && tsq < t256) return FwdForm::SQUARE_128;
  if (t128 < t192 && t128 < t256) return FwdForm::ROWS_128;
  return t192 < t256 ? FwdForm::ROWS_192 : FwdForm::ROWS_256;
}

// Backward products with K-major weights: 128 x 128 tiles, two at a time on a CU, instead of
// 256 x 256 by the same estimate; a CU's time for two of these relative to a 256 x 256 one's
// is 0.6 for dA, whose epilogues then overlap the other's MFMAs, and 0.7 for dX.  Measured as
// above, 256 x 256 against 128 x 128: dA of 8 experts x 600 rows, d 2048, h 1024 61 and 44,
// 64 x 160 143 and 119, x 256 148 and 150, x 512 210 and 234, 24 x 400, d 1024, h 1024 47 and
// 53; dX 8 x 128 63 and 40, 64 x 128 175 and 165, x 256 191 and 219.
inline bool bwd_rows_half(const RowsOf& r, int width, bool dA) {
  const int nt = (width + 255) / 256, nt128 = (width + 127) / 128;
  return !rows_stream(r, nt) &&
         (dA ? 0.6 : 0.7) * tile_rounds(r, 128, nt128, 512) < tile_rounds(r, 256, nt, 256);
}

// Weight gradients over packed rows.  An expert of few rows is an outer product whose
// time is its output's way to memory: tiles half as wide with one stage (69 KB of LDS, 128
// registers), two workgroups a CU, so that one's loads run beside the other's stores.
// Measured, rows spread by a factor of 1.35 to 1.65, us against 256 x 256 tiles of two
// stages, 64 experts, d 2048, h 1024: dW2 of 16 rows 71 and 60, 64 77 and 68, 128 91 and 84,
// 384 147 and 143, 512 167 and 170; dW1/dW3 16 rows 117 and 103, 64 131 and 133, 128 168 and
// 175; and where the wide tiles are few: 16 experts x 300 rows, d 1024, h 512, dW2 (128 wide
// tiles) 20.5 and 19.8, dW1/dW3 (256) 24.7 and 19.8, 8 x 500, d 2048, h 1024 (256 and 512)
// 27.7 and 28.3, 48 and 52.
inline bool dW2_half_wide(int E, long max_rows, int d, int h) {
  return max_rows <= 384l * E || (long)E * ((d + 255) / 256) * ((h + 255) / 256) <= 192;
}
inline bool dW13_half_wide(int E, long max_rows, int d, int h) {
  return max_rows <= 48l * E || (long)E * ((2 * h + 255) / 256) * ((d + 255) / 256) <= 256;
}

}  // namespace ec
