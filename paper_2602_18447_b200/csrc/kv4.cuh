// The 4-bit cache's block: the codes, scales and offsets of one (page of 16 keys, kv head), K and V together, HD / 2 x 36
// bytes in one piece. Codes stand where the attention kernel's lanes want them: lane (g, q) = (lane / 4, lane % 4) of
// a warp holds the operand rows g and g + 8 and the operand columns 2q, 2q + 1, 2q + 8, 2q + 9 of a 16 x 16 tile.
//  K codes  [16 keys][HD / 2 bytes]; within a row lane q's HD / 8 bytes are together: for each 64-channel group the codes
//           of channels 64 group + 16 q .. + 15, eight channels to a 32-bit word. Channel 2p + i of a word's eight sits in
//           nibble p + 4 i, so that one mask takes a pair of neighbouring channels out as two 16-bit halves.
//  V codes  by 16-channel tile: word of lane (g, q) and tile mt holds channels 16 mt + g (even nibbles) and 16 mt + g + 8
//           (odd nibbles) of keys 2q, 2q + 8, 2q + 1, 2q + 9 (bytes 0 .. 3), so that one mask takes two neighbouring keys of
//           one channel. One key of two channels is one byte: appending a key never reads what its neighbours wrote.
//           The 16-byte pieces of the lanes are permuted (v_chunk) so that a key's bytes lie in one 128-byte line per
//           64 channels and the lanes' 16-byte reads still meet no bank twice.
//  K scales, K offsets  fp16 [key % 8][key / 8][group];
//  V offsets and scales  fp16 [q][offsets by group, scales by group][keys 2q, 2q + 1, 2q + 8, 2q + 9].
#pragma once

#include <stdint.h>

namespace cs {

constexpr int kKv4Group = 64;          // channels that share a scale and an offset
// The attention multiplies a probability of up to 64 with a V scale in fp16: 64 x 1023.5 is its largest value.
constexpr float kKv4MaxScale = 1023.5f;

template <int HD>
struct Kv4 {
  static constexpr int kGroups = HD / kKv4Group;
  static constexpr int kCodes = 16 * HD / 2;
  static constexpr int kParams = 16 * kGroups * 2;
  static constexpr int kKScale = kCodes;
  static constexpr int kKOffset = kKScale + kParams;
  static constexpr int kVCodes = kKOffset + kParams;
  static constexpr int kVParams = kVCodes + kCodes;
  static constexpr int kBlock = kVParams + 2 * kParams;
  static_assert(kBlock % 16 == 0, "blocks are copied in 16-byte pieces");

  // byte of the word with channels d .. d + 7 (d a multiple of 8) of a key
  __host__ __device__ static constexpr int k_word(int key, int d) {
    return key * (HD / 2) + ((d % 64) / 16) * (HD / 8) + (d / 64) * 8 + ((d % 16) / 8) * 4;
  }
  __host__ __device__ static constexpr int k_param(int key, int group) {
    return (((key & 7) * 2 + (key >> 3)) * kGroups + group) * 2;
  }
  __host__ __device__ static constexpr int v_chunk(int g, int q) { return q * 8 + ((g + 2 * q) & 7); }
  // byte with channels 16 mt + g (low nibble) and 16 mt + g + 8 (high nibble) of a key, relative to the V codes
  __host__ __device__ static constexpr int v_byte(int key, int mt, int g) {
    return (mt / 4) * 512 + v_chunk(g, (key & 7) >> 1) * 16 + (mt % 4) * 4 + (key >> 3) + 2 * (key & 1);
  }
  // relative to the block
  __host__ __device__ static constexpr int v_offset(int key, int group) {
    return kVParams + ((((key & 7) >> 1) * 2 * kGroups + group) * 4 + (key & 1) + 2 * (key >> 3)) * 2;
  }
  __host__ __device__ static constexpr int v_scale(int key, int group) { return v_offset(key, group) + kGroups * 8; }
};

inline int kv4_block_bytes(int hd) { return hd == 128 ? Kv4<128>::kBlock : Kv4<64>::kBlock; }

}  // namespace cs
