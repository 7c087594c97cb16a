// Sine and cosine of a fraction of a turn.  Plain C++ (no CUDA types) so that the same function runs on the device and in a host
// unit test.
#pragma once
#include <math.h>
#include <stdint.h>

#if defined(__CUDACC__)
#define SPECVLM_TURN_HD __host__ __device__ __forceinline__
#else
#define SPECVLM_TURN_HD inline
#endif

namespace specvlm {

// 2^32 = a whole turn: reduced exactly to an eighth of a turn either way, there polynomials of degree 7 and 8, fitted for this file
// for the least maximum error (3.1e-9 and 5e-11; with their coefficients rounded to fp32, as they stand, 2.4e-8 and 6.7e-9, of
// which the sine's leading one is 2.2e-8).  Together with the roundings of the steps the polynomial that gives the sine there is
// off by at most 1.73 x 2^-24, the one that gives the cosine by 1.27 x 2^-24, over all 2^32 arguments.
SPECVLM_TURN_HD void turn_sincos(uint32_t turn, float& s, float& c) {
  const uint32_t quarter = (turn + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(turn - (quarter << 30)) * 2.3283064365386963e-10f;      // 2^-32
  const float u = x * x;
  float sn = fmaf(u, -75.40206909179688f, 81.5925521850586f);
  sn = fmaf(u, sn, -41.3416633605957f);
  sn = x * fmaf(u, sn, 6.2831854820251465f);
  float cs = fmaf(u, 59.22040557861328f, -85.44285583496094f);
  cs = fmaf(u, cs, 64.93931579589844f);
  cs = fmaf(u, cs, -19.739208221435547f);
  cs = fmaf(u, cs, 1.0f);
  const bool odd = quarter & 1u;
  s = odd ? cs : sn;
  c = odd ? sn : cs;
  s = quarter & 2u ? -s : s;
  c = (quarter + 1u) & 2u ? -c : c;
}

}  // namespace specvlm
