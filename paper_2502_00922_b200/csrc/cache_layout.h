// How a block of 16 tokens of one key head lies in the pool of a 4-bit cache.
//
//   keys    codes [dim / 128][16 tokens][4][<= 4] words, scales [16 tokens][groups, to even] fp16, offsets likewise
//   values  codes [dim / 64][32 lanes][<= 4] words, scales [4][groups][4] fp16, offsets likewise
//
// The order is that of the matrix instruction's A operand (16 x 16 values, two to a register), so that a lane's registers are words as
// they lie, shifted and masked: a code c in the low bits of a half is the fp16 number c 2^-24, four bits further up 16 c 2^-24.
//
// Keys: a row of the operand is a token, its columns are channels.  A word has the eight channels 8 t .. 8 t + 7 of a group (t = 0..3) of one
// token, channel c at bit 16 (c & 1) + 4 (c >> 1): four masks give the pairs (0,1), (2,3), (4,5), (6,7).
// Values: a row is a channel, the columns are tokens.  The word of lane 4 g + t for channels 16 j .. 16 j + 15 has channels 16 j + g (low
// four bits of a byte) and 16 j + g + 8 (high) of the tokens 2 t, 2 t + 8, 2 t + 1, 2 t + 9, a byte each: no byte is two tokens'.
// Scales and offsets of values: of the tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9, as the B operand's lanes want them.
#pragma once
#include <cstdint>

#include "host_device.h"

namespace huffllm {

constexpr uint32_t kCacheBlock = 16;      // tokens of a block
constexpr uint32_t kCacheGroup = 32;      // channels that share scale and offset

HUFFLLM_HD constexpr uint32_t cache_groups(uint32_t dim) { return dim / kCacheGroup; }
HUFFLLM_HD constexpr uint32_t cache_groups_even(uint32_t dim) { return (dim / kCacheGroup + 1) / 2 * 2; }
HUFFLLM_HD constexpr uint32_t cache_code_bytes(uint32_t dim) { return kCacheBlock * dim / 2; }
HUFFLLM_HD constexpr uint32_t cache_key_bytes(uint32_t dim) { return cache_code_bytes(dim) + kCacheBlock * cache_groups_even(dim) * 4; }
HUFFLLM_HD constexpr uint32_t cache_block_bytes(uint32_t dim) { return cache_key_bytes(dim) + cache_code_bytes(dim) + kCacheBlock * cache_groups(dim) * 4; }

// Bytes into a block: the word of keys with channels 32 group + 8 t .. of token r
HUFFLLM_HD constexpr uint32_t key_word_at(uint32_t dim, uint32_t r, uint32_t group, uint32_t t) {
    const uint32_t part = group / 4, rest = cache_groups(dim) - 4 * part, words = rest < 4 ? rest : 4;
    return part * 1024 + ((r * 4 + t) * words + group % 4) * 4;
}
HUFFLLM_HD constexpr uint32_t key_scale_at(uint32_t dim, uint32_t r, uint32_t group) { return cache_code_bytes(dim) + (r * cache_groups_even(dim) + group) * 2; }
HUFFLLM_HD constexpr uint32_t key_offset_at(uint32_t dim, uint32_t r, uint32_t group) {
    return key_scale_at(dim, r, group) + kCacheBlock * cache_groups_even(dim) * 2;
}
// The byte of values with channel d (d / 8 even: low four bits, and channel d + 8 in the high ones) of token r
HUFFLLM_HD constexpr uint32_t value_byte_at(uint32_t dim, uint32_t r, uint32_t d) {
    const uint32_t j = d / 16, part = j / 4, rest = dim / 16 - 4 * part, words = rest < 4 ? rest : 4, lane = d % 8 * 4 + r % 8 / 2;
    return cache_key_bytes(dim) + part * 512 + (lane * words + j % 4) * 4 + r % 2 * 2 + r / 8;
}
HUFFLLM_HD constexpr uint32_t value_scale_at(uint32_t dim, uint32_t r, uint32_t group) {
    return cache_key_bytes(dim) + cache_code_bytes(dim) + ((r % 8 / 2 * cache_groups(dim) + group) * 4 + r % 2 + r / 8 * 2) * 2;
}
HUFFLLM_HD constexpr uint32_t value_offset_at(uint32_t dim, uint32_t r, uint32_t group) { return value_scale_at(dim, r, group) + kCacheBlock * cache_groups(dim) * 2; }

}  // namespace huffllm
