// Keys of the routing kernels (sdp_route.hip), free of HIP so that they can be
// checked without a device.  A key is a float whose last four bits say where in its
// lane the expert is, so that a lane's keys are sorted by maxima and minima alone.
#pragma once

#include <cstdint>

namespace sdpops {

constexpr uint32_t kPlace = 15;

constexpr uint32_t key_bits(float v) { return __builtin_bit_cast(uint32_t, v); }
constexpr float key_with(float v, uint32_t place) {
    return __builtin_bit_cast(float, (key_bits(v) & ~kPlace) | place);
}
constexpr float without_place(float key) { return key_with(key, 0); }

// The key of value v of a lane's i-th expert.  EXACT: v has nothing in its last four
// bits, and among equals the lowest i has the largest key; -0 counts as 0 (it loses its
// sign before the sign says which way places count).  Minus infinity stays what it is.
template <bool EXACT>
constexpr float key_of(float v, uint32_t i) {
    const float k = EXACT ? v + 0.0f : v;
    if (k == -__builtin_huge_valf()) return k;
    return key_with(k, EXACT && key_bits(k) >> 31 ? i : kPlace - i);
}
// i of such a key.
template <bool EXACT>
constexpr uint32_t place_of(float key) {
    const uint32_t bits = key_bits(key);
    return (EXACT && bits >> 31 ? bits : ~bits) & kPlace;
}

// Half of a group's worth, of its two best keys (or one; minus infinity: not there), and
// how far it may be from that of the scores and biases themselves.  (The sum of two lowest
// values, or of two largest ones, is past FP32; half of it is not.)  A key's four bits, its sum with
// the bias and the worth's own addition are 33 roundings in proportion to the keys, which
// may cancel in the worth; the scores, the sum of a softmax most of them, are off by 40
// roundings of one.  (Taken as 48 of each.)
struct Worth {
    float value, room;
};
constexpr float size_of(float v) { return v < 0.0f ? -v : v; }
constexpr Worth worth_of(float first, float second) {
    constexpr float kNone = -__builtin_huge_valf();
    if (first == kNone) return {kNone, 0.0f};
    if (second == kNone) second = 0.0f;
    return {0.5f * first + 0.5f * second, (0.5f + 0.5f * size_of(first) + 0.5f * size_of(second)) * 0x1.8p-19f};
}

}  // namespace sdpops
