// Byte order of a page: 64 tokens of one head, codes of head_dim values each, in the order in which
// the attention's matrix instructions take them (16x16x32, lane l: row or column l % 16, values
// 8 (l / 16) .. + 7 of the 32), two fragments to a lane's 16-byte load.  Host and device.
//   keys    [pair of 16 tokens: 2][dims / 32][lane][2 x 8]: token 32 p + 16 (e / 8) + lane % 16,
//           dim 32 k + 8 (lane / 16) + e % 8
//   values  [dims / 16][lane][2 x 8]: dim 16 t + lane % 16, token 32 (e / 8) + 16 (e % 8 / 4)
//           + 4 (lane / 16) + e % 4: the tokens whose scores the lane holds, in its registers' order
#pragma once

#ifdef __HIPCC__
#define TMZ_HD __host__ __device__
#else
#define TMZ_HD
#endif

namespace tmz {

constexpr int kBlock = 64;            // tokens of a block

template <int HD>
TMZ_HD constexpr int key_at(int t, int d) {
  return (((t >> 5) * (HD / 32) + (d >> 5)) * 64 + ((t & 15) | (((d >> 3) & 3) << 4))) * 16 +
         ((t >> 4 & 1) << 3) + (d & 7);
}
TMZ_HD constexpr int value_at(int t, int d) {
  return ((d >> 4) * 64 + ((d & 15) | (((t & 15) >> 2) << 4))) * 16 + ((t >> 5) << 3) +
         ((t >> 4 & 1) << 2) + (t & 3);
}

}  // namespace tmz
