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

}  // namespace ec
