// The 4-bit format of cached rows: a sign, two exponent bits and one of mantissa, and a power-of-two scale for 32 channels.
// The same code on the host, where it is compared with the definition.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define AA_HD __host__ __device__ __forceinline__
#else
#define AA_HD inline
#endif

namespace aa {

constexpr int kFp4Group = 32;               // channels with one scale

// `top`: the bits of the largest magnitude of a group, as of a float (NaN above infinity above numbers).
// The scale byte: 127 + the least e of [-120, 125] with top <= 7 * 2^e, or 255 if the group holds a NaN or an infinity.
// 7: a largest value between 6 and 7 loses less by being cut to 6 than the group loses by the next coarser scale (root mean square
// error of normal values 0.1119; with 6 0.1154, with 8 0.1150; heavier tails 0.129 / 0.139 / 0.131).
// The bounds keep every code's value a normal bf16 number.
AA_HD int fp4_scale_byte(uint32_t top) {
    const int ex = (int)(top >> 23);
    if (ex == 255) return 255;
    const int e = ex - 127 - 2 + ((top & 0x7fffffu) > 0x600000u);
    return 127 + (e < -120 ? -120 : e > 125 ? 125 : e);
}

}  // namespace aa
