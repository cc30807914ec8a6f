// Launchers of the 8-bit activation checkpoints (ckpt8.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_common.h"

namespace libra {

// Four packed tensors and the bf16 buffers that they are unpacked into; chunks: elements / 16.
struct Ckpt8Four {
  const int8_t *q[4];
  const uint8_t *e[4];
  bf16 *x[4];
  int64_t chunks[4];
};

int launch_ckpt8_pack(const void *x, bool fp32, int64_t rows, int64_t cols, int64_t ld, int8_t *q,
                      uint8_t *e, hipStream_t st);
int launch_ckpt8_unpack(const int8_t *q, const uint8_t *e, int64_t rows, int64_t cols, bool fp32,
                        int64_t ld, void *x, hipStream_t st);
int launch_ckpt8_unpack4(const Ckpt8Four &a, hipStream_t st);

}  // namespace libra
