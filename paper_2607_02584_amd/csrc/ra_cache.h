// ra_cache.h -- layout of the 4-bit paged KV cache and what its kernels share
// (library-internal).
//
// A page of `page` tokens holds, head after head, one block of page * (D + 8)
// bytes: K codes, V codes (page * D / 2 each), K scales, V scales (binary32,
// one per token).  Every block begins on 128 bytes (page is a multiple of 16).
//
// Codes are E2M1 floats (sign, 2 exponent bits, 1 mantissa bit: 0, .5, 1, 1.5,
// 2, 3, 4, 6): gfx950 turns a byte of two of them into two 16-bit floats with
// one instruction and no bias to take off afterwards, where integers in
// nibbles take a shift, a mask and a correction, and on rotated (near normal)
// values both have the same error (0.11 of the standard deviation).
//
// The order of the codes makes 16 tokens of a head operands of the 16x16x32
// matrix product as they lie in memory, D / 8 bytes per lane, whole wave
// loads being contiguous:
//   K: [tile of 16 tokens][part of D/4 channels][token][D/8 bytes]   lane = part * 16 + token
//   V: [group of 4 tokens][16 chunks of D/16 channels][token][D/32 bytes]   lane = group * 16 + chunk
// A token's codes are whole bytes of their own, so tokens are written without
// reading what lies beside them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace ra {

struct CacheGeom {
  uint8_t* cache;
  int64_t page_bytes;
  int num_pages, page, page_log, Hkv;
};

template <int D>
__host__ __device__ constexpr int head_bytes(int page) { return page * (D + 8); }

// ---- arguments ----
struct PlanArgs {
  const int* seq_lens;
  const int* new_lens;
  const int* release;    // [R] or nullptr
  int* block_table;      // [R][max_blocks]
  int* free_pages;       // [num_pages], the top of the stack at free_count - 1
  const int* free_count;
  int* seq_out;
  int* count_out;
  int* q_start;          // [R + 1]
  int* positions;        // [T]
  int* slots;            // [T]
  int* status;           // [4]
  int R, T, max_blocks, num_pages, page, page_log;
};

struct AppendArgs {
  CacheGeom g;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_ts, k_hs, v_ts, v_hs;   // token and head strides, elements
  const int* slots;
  const int* positions;
  const float* rope;                // [rope_rows][D/2][2] or nullptr
  int rope_rows, T, is_fp16, heads; // heads: KV heads per workgroup
};

struct ReadArgs {
  CacheGeom g;
  const int* slots;
  void* k;                          // [T][Hkv][D]
  void* v;
  int T, out_dtype, heads;
};

struct CacheAttnArgs {
  CacheGeom g;
  const uint16_t* q;
  int64_t q_ts, q_hs;
  const int* block_table;
  const int* q_start;
  const int* seq_lens;
  const float* rope;
  void* o;                          // [T][Hq][D]
  float* lse;                       // [T][Hq] or nullptr
  float* part_o;                    // partial outputs of split rows
  float2* part_ml;                  // their running maxima and sums
  float c;                          // softmax scale * log2(e), and 1/sqrt(D) where Q is rotated
  int rope_rows, R, T, max_q, Hq, G, max_blocks;
  int causal, window, is_fp16, out_dtype, had, vhad;
  int target, target_rows;          // pieces of work per KV head aimed at (set by the launch)
  // first tokens that stay visible beside a window; partial rows of few rows beside those of many
  int sinks;
  float* few_o;
  float2* few_ml;
  // prefixes that requests share
  int groups;
  const int* group_start;           // [groups + 1]
  const int* prefix_lens;           // [groups]
  const int* positions;             // [T]
  // set by the launch
  int4* requests;                   // [groups + R][2] prefixes and requests
  int2* info;                       // [groups + R] where their parts are: first row, parts (negative: from the back)
  int2* owner;                      // [T] request and group of a token
  int4* pieces[2];                  // of few and of many rows
  int* counts;                      // [2]
  int bound[2];                     // of the pieces
  uint16_t* turned;                 // [T][Hq][2][D] Q as the matrix products of few rows take it
  uint8_t* turned6;                 // [T][Hq][5][D] in 6 bits each, of many rows
  float* back;                      // [T][Hq] what the scores are multiplied by
  int64_t part_rows;                // rows of part_o for each KV head
};

hipError_t launch_cache_plan(const PlanArgs& a, hipStream_t s);
hipError_t launch_cache_append(const AppendArgs& a, int D, bool hadk, bool hadv, hipStream_t s);
hipError_t launch_cache_read(const ReadArgs& a, int D, bool hadk, bool hadv, hipStream_t s);
hipError_t launch_cache_attn(const CacheAttnArgs& a, int D, hipStream_t s);
hipError_t launch_cache_attn_sinks(const CacheAttnArgs& a, int D, hipStream_t s);
hipError_t launch_cache_attn_shared(const CacheAttnArgs& a, int D, void* workspace, hipStream_t s);
size_t cache_shared_bytes(int D, int Hkv, int G, int R, int groups, int T);
// bytes of workspace that launch_cache_attn's part_o and part_ml take
size_t cache_attn_partial_bytes(int D, int Hkv, int G, int max_q, size_t* ml_offset);
// of cache_attn_sinks, which is not less, and where the partial rows of requests of few rows lie
size_t cache_sinks_bytes(int D, int Hkv, int G, int max_q, size_t* ml, size_t* few_o, size_t* few_ml);

// stores a library error message for rotate_attn_last_error() and returns code
int set_error(int code, const char* msg) noexcept;

// ---- lanes ----
// The value of lane ^ M (M = 1, 2, 7, 8: one register move inside a row of 16, 4: two).
template <int M>
__device__ __forceinline__ int lane_xor(int v) {
  if constexpr (M == 1) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);    // quad_perm 1,0,3,2
  if constexpr (M == 2) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);    // quad_perm 2,3,0,1
  if constexpr (M == 4)                                                              // half mirror (^7), then ^3
    return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);
  if constexpr (M == 7) return __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);   // half mirror
  if constexpr (M == 8) return __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true);   // row_ror:8
  if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (__lane_id() & 16) ? r[0] : r[1];
  }
  if constexpr (M == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (__lane_id() & 32) ? r[0] : r[1];
  }
}
template <int M>
__device__ __forceinline__ float lane_xor(float v) {
  return __int_as_float(lane_xor<M>(__float_as_int(v)));
}
template <int M>
__device__ __forceinline__ double lane_xor(double v) {
  return __hiloint2double(lane_xor<M>(__double2hiint(v)), lane_xor<M>(__double2loint(v)));
}

// x's value of the lanes with bit M and y's of those without it change places.
template <int M>
__device__ __forceinline__ void lane_swap(float& x, float& y) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t u = __float_as_uint(x), v = __float_as_uint(y);
  const auto z = [&] {
    if constexpr (M == 32) return __builtin_amdgcn_permlane32_swap(u, v, false, false);
    else return __builtin_amdgcn_permlane16_swap(u, v, false, false);
  }();
  x = __uint_as_float(z[0]);
  y = __uint_as_float(z[1]);
#endif
}
// One butterfly stage between lanes that differ in bit M.  Where halves of a wave or of 32 lanes are exchanged,
// two values at a time: a lane takes both sides of one of them, and gives back what is the other's.
template <int M, typename F, int N>
__device__ __forceinline__ void butterfly_lanes(F (&y)[N], int lane) {
  if constexpr (sizeof(F) == 4 && M >= 16 && N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      F a = y[i], b = y[i + 1];
      lane_swap<M>(a, b);
      y[i] = a + b;
      y[i + 1] = a - b;
      lane_swap<M>(y[i], y[i + 1]);
    }
    return;
  }
  const bool up = lane & M;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const F o = lane_xor<M>(y[i]);
    y[i] = o + (up ? -y[i] : y[i]);
  }
}
// The stages inside a lane's N values.
template <typename F, int N>
__device__ __forceinline__ void butterfly_regs(F (&y)[N]) {
#pragma unroll
  for (int h = 1; h < N; h *= 2)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(i & h)) {
        const F a = y[i], b = y[i + h];
        y[i] = a + b;
        y[i + h] = a - b;
      }
}

// ---- rows of D channels, 8 per lane ----
//
// D / 8 lanes hold a row.  Lane l holds channels 8 b .., b = row_block(l): with
// this order the three low lane stages of the Hadamard transform exchange with
// lanes ^ 1, ^ 2 and ^ 7, each one register move (^ 4 would take two).
__device__ __forceinline__ int row_block(int lane) { return lane ^ ((lane & 4) ? 3 : 0); }

// y + s * (y of the partner lane), a stage of eight values: one multiply-add
// each that takes its factor through the move (the compiler makes two
// operations of it).  Values written just before need two wait states ahead of
// such a move.
#if defined(__HIP_DEVICE_COMPILE__)
#define RA_STAGE8(move)                                                                                            \
  asm volatile("s_nop 1\n\t"                                                                                       \
               "v_fmac_f32_dpp %0, %0, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %1, %1, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %2, %2, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %3, %3, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %4, %4, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %5, %5, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %6, %6, %8 " move " row_mask:0xf bank_mask:0xf\n\t"                                 \
               "v_fmac_f32_dpp %7, %7, %8 " move " row_mask:0xf bank_mask:0xf"                                      \
               : "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]), "+v"(y[4]), "+v"(y[5]), "+v"(y[6]), "+v"(y[7])     \
               : "v"(s))
#else
#define RA_STAGE8(move) (void)s
#endif
template <int M>
__device__ __forceinline__ void stage8(float (&y)[8], bool up) {
  const float s = up ? -1.0f : 1.0f;
  if constexpr (M == 1) RA_STAGE8("quad_perm:[1,0,3,2]");
  if constexpr (M == 2) RA_STAGE8("quad_perm:[2,3,0,1]");
  if constexpr (M == 7) RA_STAGE8("row_half_mirror");
  if constexpr (M == 8) RA_STAGE8("row_ror:8");
}

// Times the Sylvester-Hadamard matrix of +-1, and times row_sign(b): a stage is
// y + s o with s = -1 in lanes whose bit is set, where o - y is meant, a sign
// that all later partners share.
template <int D>
__device__ __forceinline__ void hadamard_row(float (&y)[8], int b) {
  butterfly_regs(y);
  stage8<1>(y, b & 1);
  stage8<2>(y, b & 2);
  stage8<7>(y, b & 4);
  if constexpr (D == 128) stage8<8>(y, b & 8);
}
__device__ __forceinline__ float row_sign(int b) { return __builtin_popcount(b) & 1 ? -1.0f : 1.0f; }
// The same in binary64, without the sign.
template <int D>
__device__ __forceinline__ void hadamard_row(double (&y)[8], int b) {
  butterfly_regs(y);
  auto stage = [&](auto mm, bool up) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = lane_xor<decltype(mm)::value>(y[i]) + (up ? -y[i] : y[i]);
  };
  stage(std::integral_constant<int, 1>{}, b & 1);
  stage(std::integral_constant<int, 2>{}, b & 2);
  stage(std::integral_constant<int, 7>{}, b & 4);
  if constexpr (D == 128) stage(std::integral_constant<int, 8>{}, b & 8);
}

// ---- 16-bit values ----
__device__ __forceinline__ float cache_h2f(uint16_t b, int is_fp16) {
  return is_fp16 ? static_cast<float>(__builtin_bit_cast(_Float16, b)) : __uint_as_float(static_cast<uint32_t>(b) << 16);
}
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
// two binary32 values, each rounded once to nearest even
__device__ __forceinline__ uint32_t pack16(float a, float b, bool fp16) {
  if (fp16) {
    const v2h r = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
    return __builtin_bit_cast(uint32_t, r);
  }
  const v2bf r = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, r);
}

}  // namespace ra
