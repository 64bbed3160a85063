// csrc/philox.h as the device compiles it, for the host.
#include "philox.h"

extern "C" void philox(const uint32_t* c, const uint32_t* k, uint32_t* out) {
  const moe::Philox4 r = moe::philox4x32_10(c[0], c[1], c[2], c[3], k[0], k[1]);
  for (int i = 0; i < 4; ++i) out[i] = r.w[i];
}
