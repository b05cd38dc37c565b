// Driver for an AddressSanitizer + UndefinedBehaviorSanitizer build of the vocabulary head's HOST code: argument checks, plans,
// workspace arithmetic.  Every call is one that the host rejects, or that has nothing to enqueue, so it runs without a GPU.
// Exit code 0 and no sanitizer report is the test (tests/test_sanitizers_head_cpu.py builds and runs it).
#include <climits>
#include <cstdint>
#include <cstdio>
#include <vector>

#include "sip_head.h"

static int fails = 0;
#define EXPECT(cond)                                                                            \
  do {                                                                                          \
    if (!(cond)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #cond); ++fails; }           \
  } while (0)

int main() {
  void* dev = reinterpret_cast<void*>(0x100000);
  const int32_t* di = reinterpret_cast<const int32_t*>(0x200000);
  float* df = reinterpret_cast<float*>(0x300000);
  uint8_t* db = reinterpret_cast<uint8_t*>(0x400000);
  const int32_t counts[] = {INT32_MIN, -1, 0, 1, 63, 64, 65, 300, 8192, 65535, 65536, 65537, INT32_MAX};
  const int32_t vocabularies[] = {INT32_MIN, -5, 0, 1, 255, 257, 32000, 151643, SIP_MAX_V, SIP_MAX_V + 1, INT32_MAX};
  const int32_t widths[] = {INT32_MIN, -8, 0, 1, 7, 8, 32, 2080, 4096, SIP_MAX_D, SIP_MAX_D + 8, INT32_MAX - 7};
  const int64_t strides[] = {INT64_MIN, -8, 0, 1, 8, 4096, 1 << 20, (int64_t)1 << 30, (int64_t)1 << 33, INT64_MAX - 7, INT64_MAX};

  // cross entropy: sizes, plans of every shape (a backward pass without gradients plans, and enqueues nothing), rejected calls
  for (int32_t N : counts)
    for (int32_t V : vocabularies)
      for (int32_t D : widths) {
        const size_t one = sip_xent_workspace_bytes(N, V, D, 0), both = sip_xent_workspace_bytes(N, V, D, 1);
        const bool ok = N > 0 && V > 0 && D > 0 && D % 8 == 0 && N <= SIP_MAX_TOKENS && V <= SIP_MAX_V && D <= SIP_MAX_D;
        EXPECT((one > 0) == ok && (both >= one) && one % 256 == 0 && both % 256 == 0);
        const sip_status st = sip_xent_backward(dev, N, D, D, dev, V, D, di, 1.0f, df, df, nullptr, 1.0f, nullptr, 0, nullptr, 0, dev, both, nullptr);
        EXPECT(ok ? st == SIP_OK : (st == SIP_ERR_INVALID_ARG || st == SIP_ERR_UNSUPPORTED));
        if (ok)
          for (int64_t s : strides) {
            EXPECT(sip_xent_forward(dev, N, D, s, dev, V, D, di, 1.0f, df, df, nullptr, 0, nullptr) != SIP_OK);
            EXPECT(sip_xent_forward(dev, N, D, D, dev, V, s, di, 1.0f, df, df, nullptr, 0, nullptr) != SIP_OK);
            EXPECT(sip_xent_backward(dev, N, D, D, dev, V, D, di, 1.0f, df, df, nullptr, 1.0f, dev, s, dev, s, nullptr, 0, nullptr) != SIP_OK);
          }
      }

  // 4-bit head
  for (int32_t B : {INT32_MIN, -1, 0, 1, 16, 64, 65, 256, 1 << 20, INT32_MAX})
    for (int32_t V : vocabularies)
      for (int32_t D : widths)
        for (int32_t group : {INT32_MIN, 0, 16, 32, 64, 128, 256}) {
          const size_t need = sip_head_workspace_bytes(B, V, D, group);
          EXPECT(need % 256 == 0);
          for (int64_t s : strides)
            for (sip_dtype x : {SIP_F32, SIP_BF16}) {
              EXPECT(sip_head_logits(dev, B, D, s, x, db, D / 2, dev, x, nullptr, group, V, dev, V, x, nullptr, need, nullptr) != SIP_OK);
              EXPECT(sip_head_logits(dev, B, D, D, x, db, s, dev, x, db, group, V, dev, s, x, nullptr, need, nullptr) != SIP_OK);
              EXPECT(sip_head_quantize(dev, V, D, s, group, db, D / 2, nullptr, x, nullptr, nullptr) != SIP_OK);
              EXPECT(sip_head_quantize(reinterpret_cast<void*>(0x100002), V, D, D, group, db, s, dev, x, db, nullptr) != SIP_OK);
            }
        }

  // clipping
  for (int32_t n : counts) EXPECT((sip_grad_clip_workspace_bytes(n) > 0) == (n >= 0 && n <= SIP_MAX_TENSORS));
  for (int64_t count : {INT64_MIN, (int64_t)-1, (int64_t)0, (int64_t)7, (int64_t)1 << 40, ((int64_t)1 << 40) + 1, INT64_MAX})
    for (int32_t n : {1, 120, 121, SIP_MAX_TENSORS}) {
      std::vector<sip_grad> table(n, sip_grad{dev, dev, count, n & 1 ? SIP_BF16 : SIP_F32});
      EXPECT(sip_grad_clip(table.data(), n, 1.0f, 0.0f, df, nullptr, 0, nullptr) != SIP_OK);
      EXPECT(sip_grad_clip(table.data(), n, 1.0f, 0.0f, df, dev, sip_grad_clip_workspace_bytes(n) - 1, nullptr) != SIP_OK);
    }
  EXPECT(sip_grad_clip(nullptr, 1, 1.0f, 0.0f, df, dev, 1 << 20, nullptr) == SIP_ERR_INVALID_ARG);
  EXPECT(sip_grad_clip(nullptr, INT32_MAX, 1.0f, 0.0f, df, dev, 1 << 20, nullptr) != SIP_OK);

  if (fails) return 1;
  std::puts("ok");
  return 0;
}
