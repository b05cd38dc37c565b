// Driver for an AddressSanitizer + UndefinedBehaviorSanitizer build of the HOST code of beams, adapters and embedding: argument checks and
// workspace arithmetic.  Every call is one that the host rejects, or that has nothing to enqueue, so it runs without a GPU.
// Exit code 0 and no sanitizer report is the test (tests/test_sanitizers_search_cpu.py builds and runs it).
#include <climits>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "sip_beam.h"
#include "sip_head.h"

static int fails = 0;
#define EXPECT(cond)                                                                            \
  do {                                                                                          \
    if (!(cond)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond); ++fails; }           \
  } while (0)

int main() {
  void* dev = reinterpret_cast<void*>(0x100000);
  int32_t* di = reinterpret_cast<int32_t*>(0x200000);
  float* df = reinterpret_cast<float*>(0x300000);
  uint8_t* db = reinterpret_cast<uint8_t*>(0x400000);
  const int32_t counts[] = {INT32_MIN, -1, 0, 1, 63, 64, 65, 300, 8192, 65535, 65536, 65537, 1 << 20, INT32_MAX};
  const int32_t vocabularies[] = {INT32_MIN, -5, 0, 1, 255, 8193, 32000, 151643, SIP_MAX_V, SIP_MAX_V + 1, INT32_MAX};
  const int32_t widths[] = {INT32_MIN, -8, 0, 1, 7, 8, 32, 2080, 4096, SIP_MAX_D, SIP_MAX_D + 8, INT32_MAX - 7};
  const int64_t strides[] = {INT64_MIN, -8, 0, 1, 8, 4096, 1 << 20, (int64_t)1 << 30, (int64_t)1 << 33, INT64_MAX - 7, INT64_MAX};

  for (int32_t groups : counts)
    for (int32_t width : {INT32_MIN, -1, 0, 1, 4, 64, 65, INT32_MAX})
      for (int32_t V : vocabularies)
        for (int32_t n : {INT32_MIN, 0, 1, 8, 128, 129, INT32_MAX}) {
          const size_t need = sip_beam_workspace_bytes(groups, width, V, n);
          const bool ok = groups > 0 && width > 0 && width <= 64 && V > 0 && V <= SIP_MAX_V && n > 0 && n <= 128 &&
                          (int64_t)groups * width <= SIP_MAX_B;
          EXPECT((need > 0) == ok && need % 256 == 0);
          for (int64_t s : strides)
            for (sip_dtype t : {SIP_F32, SIP_BF16}) {
              EXPECT(sip_beam_select(dev, groups, width, V, s, t, 1.0f, df, db, V - (V > INT32_MIN), df, n, di, di, df, nullptr, need, nullptr) != SIP_OK);
              EXPECT(sip_beam_select(dev, groups, width, V, s, t, 0.0f, df, nullptr, 0, nullptr, n, di, di, df, dev, need, nullptr) == SIP_ERR_INVALID_ARG);
            }
        }
  for (int32_t slots : counts)
    for (int32_t L : {INT32_MIN, 0, 1, 100, SIP_MAX_L, SIP_MAX_L + 1, INT32_MAX})
      for (int32_t groups : counts)
        for (int32_t width : {INT32_MIN, 0, 1, 64, 65, INT32_MAX})
          EXPECT(sip_state_reorder(nullptr, SIZE_MAX, slots, L, groups, width, di, di, di, nullptr) != SIP_OK);

  for (int32_t N : counts)
    for (int32_t V : vocabularies)
      for (int32_t D : widths) {
        const size_t need = sip_embed_workspace_bytes(N, V, D);
        const bool ok = N >= 0 && N <= SIP_MAX_TOKENS && V > 0 && V <= SIP_MAX_V && D > 0 && D % 8 == 0 && D <= SIP_MAX_D;
        EXPECT((need > 0) == ok && need % 256 == 0);
        const sip_status nothing = sip_embed_backward(dev, D, SIP_F32, di, 0, V, D, 1.0f, 1, dev, D, SIP_BF16, dev, SIZE_MAX, nullptr);
        EXPECT((nothing == SIP_OK) == (V > 0 && V <= SIP_MAX_V && D > 0 && D % 8 == 0 && D <= SIP_MAX_D));
        for (int64_t s : strides) {
          EXPECT(sip_embed_backward(dev, s, SIP_BF16, di, N, V, D, 1.0f, 0, dev, s, SIP_F32, nullptr, need, nullptr) != SIP_OK);
          EXPECT(sip_embed(reinterpret_cast<void*>(0x100004), SIP_F32, V, D, s, di, N, 1.0f, dev, s, SIP_F32, nullptr) != SIP_OK);
          EXPECT(sip_embed_codes(db, s, nullptr, SIP_F32, db, 32, V, D, di, N, 1.0f, dev, s, SIP_F32, nullptr) != SIP_OK);
          (void)sip_embed(dev, SIP_BF16, V, D, s, di, 0, 1.0f, dev, s, SIP_BF16, nullptr);
          (void)sip_embed_codes(db, s, dev, SIP_BF16, nullptr, 64, V, D, di, 0, 1.0f, dev, s, SIP_BF16, nullptr);
        }
      }
  for (int32_t B : counts)
    for (int32_t A : {INT32_MIN, 0, 1, 4096, 4097, INT32_MAX})
      for (int32_t r : {INT32_MIN, 0, 8, 12, 128, 136, INT32_MAX - 7})
        for (int32_t D : widths) {
          const size_t need = sip_head_adapt_workspace_bytes(B, A, r, D);
          EXPECT(need % 256 == 0);
          for (int64_t s : strides)
            EXPECT(sip_head_adapt(dev, B, D, s, SIP_BF16, dev, dev, A, r, di, df, 1000, dev, s, SIP_F32, nullptr, need, nullptr) != SIP_OK);
        }

  if (fails) return 1;
  std::puts("ok");
  return 0;
}
