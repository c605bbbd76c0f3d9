// Internal: caches in 8 bits.  A value is e4m3 * 2^(E - 127), E one byte for kQ8Block rows of a head.
#pragma once
#include "lsp_attn.h"

namespace lsp {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kQ8Block = LSP_Q8_BLOCK;
static_assert(kQ8Block == 32, "the kernels take blocks of 32 rows");
constexpr int kQ8Most = 246;  // the largest E: 1.75 * 2^127 is the largest magnitude then

// 2^(E - 127), E from 1 to 254
__device__ __forceinline__ float q8_scale(uint32_t E) { return __uint_as_float(E << 23); }

// Operands of the layers of one launch: 64 bytes a layer, which a workgroup reads at once (arrays of each operand were eight reads in a chain,
// 3 us of a short call).
struct Q8Layer {
  const char *q, *k_suf, *v_suf;
  char *k_cache, *v_cache;
  uint8_t *k_scale, *v_scale;
  char *out;
};
struct Q8Layers {
  Q8Layer of[kMaxAttnLayers];
};

// Shapes and strides of caches in 8 bits beside buffers of the descriptor's type, checked and resolved.
int32_t check_q8(const char *what, const lsp_attn_desc *d, bool queries, AttnArgs &a);

}  // namespace lsp
