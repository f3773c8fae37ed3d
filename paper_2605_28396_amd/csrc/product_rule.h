// Which tiles serve a product of 8-bit rows, and how its vocabulary is cut into strips (host arithmetic alone).
#pragma once
#include <stdint.h>

namespace adwin {

// Strips of the vocabulary for `tiles` token tiles: one workgroup occupies a compute unit, so that what counts is the number of
// rounds times the tiles of the longest strip (*turns); of as good ones in a single round the most.  A launch has fewer than 2^32 threads.
inline int product_strips(int64_t tiles, int32_t vocab_tiles, int64_t* turns = nullptr) {
  int64_t best = 0;
  int strips = 1;
  for (int s = 1; s <= vocab_tiles && s <= 256; ++s) {
    if (s > 1 && tiles * s * 256 >= (int64_t)1 << 32) break;
    const int64_t cost = (tiles * s + 255) / 256 * ((vocab_tiles + s - 1) / s);
    if (best == 0 || cost < best || (cost == best && tiles * s <= 256)) { best = cost; strips = s; }
  }
  if (turns) *turns = best;
  return strips;
}

// The tile of a product: 256 tokens x 256 entries (0), 64 x 128 (1) or 128 x 128 (2).
struct ProductWay {
  int tokens, entries;
  double first;                    // the launches' ends, the tokens' integers among them
  double tile, step;               // of a tile and of a k-step, `turns` tiles one after the other on the busiest compute unit
  double w, z;                     // of a megabyte of the head and of the logits, what the steps do not cover
};
constexpr ProductWay kProductWays[3] = {
    {256, 256, 9.9, 4.96, 1.29, 0.075, 0.195}, {64, 128, 7.1, 1.06, 0.42, 0.050, 0.233}, {128, 128, 7.6, 1.23, 0.595, 0.038, 0.225}};

// us that a call takes in this way
inline double product_us(const ProductWay& p, int64_t T, int32_t V, int pitch, int z_bytes) {
  int64_t turns;
  product_strips((T + p.tokens - 1) / p.tokens, (V + p.entries - 1) / p.entries, &turns);
  return p.first + (double)turns * (p.tile + pitch / 128 * p.step) + 1e-6 * ((double)V * pitch * p.w + (double)T * V * z_bytes * p.z);
}

// Fitted to 373 calls of 65 to 8,200 tokens, V = 500 to 151,936, H = 100 to 4096, each measured in the three ways: off by 9 % (rms) and 49 % at
// most (V = 902), and the way that it takes is within 4 % of the fastest, by 0.1 % on average.  Of 90 calls that it had not seen (off by 11 %,
// 32 % at most) it takes one 11 % and one 7 % slower than the fastest, the others within 4 %.
// us, 256 x 256 / 64 x 128 / 128 x 128: 1,000 tokens, V = 2,000, H = 1024 25.5 / 12.7 / 14.6; V = 8,000, H = 2048
// 39.3 / 39.5 / 32.6; 400 tokens, V = 32,000, H = 1024 28.8 / 40.3 / 34.6; 600 tokens, V = 50,000 71.0 / 93.4 / 73.2; 2,048 tokens, V = 16,000,
// H = 2048 80.9 / 152 / 114; 192 tokens, V = 75,000 79.9 / 77.6 / 71.8; V = 151,936: 100 tokens, H = 4096 200 / 190 / 172, 192 tokens
// 211 / 248 / 232, 300 tokens, H = 1024 112 / 139 / 111.
inline int product_tile(int64_t T, int32_t V, int pitch, int z_bytes) {
  int best = 0;
  double least = 0;
  for (int i = 0; i < 3; ++i) {
    const double us = product_us(kProductWays[i], T, V, pitch, z_bytes);
    if (i == 0 || us < least) { least = us; best = i; }
  }
  return best;
}

}  // namespace adwin
