// The packed form of matrices in microscaled 4-bit floating point, as their writers and the two head kernels see it.
//
// An element is one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign; a group of columns of a row shares a scale:
//   groups of 32: a power of two, held as its exponent in a byte
//   groups of 16: a number of four exponent and three mantissa bits, times a power of two common to the whole matrix (weights) or to
//                 the row (activations), which uses the range of those bits whatever the magnitude of the values
// The tensor core (kind::mxf4nvf4) multiplies two matrices of this form, scales and all.
//
// A unit holds 128 rows (a weight tile; fewer for a narrow tile of activations) and 128 columns, as the tensor core reads them:
//   scales    512 bytes per 64 columns (groups of 16) or per 128 (groups of 32): row r's four in the word (r % 32) * 4 + r / 32, which one
//             copy to tensor memory brings into place
//   elements  64 bytes per row, column 2i in the low half of byte i; the four 16-byte parts of row r are permuted by (r / 2) % 4 (the
//             64-byte swizzle of shared memory), rows and all ready for a plain bulk copy
// and the units of a row tile lie one behind the other.  Columns beyond d are zeros.
#pragma once

#include "common.cuh"
#include "sm100_operands.cuh"

namespace ee {

constexpr int kFp4Rows = 128;                    // of a weight tile
constexpr int kFp4Cols = 128;                    // of a unit
constexpr int kFp4Header = 256;                  // packed weights begin with the power of two they have in common (fp32)

__host__ __device__ constexpr int fp4_scale_bytes(int group) { return group == 16 ? 1024 : 512; }      // of a unit
__host__ __device__ constexpr int fp4_unit_bytes(int group, int rows) { return fp4_scale_bytes(group) + rows * (kFp4Cols / 2); }
__host__ __device__ inline int fp4_blocks(int d) { return (d + kFp4Cols - 1) / kFp4Cols; }
__host__ __device__ inline int fp4_tiles(int n, int rows) { return (n + rows - 1) / rows; }

// Where row r of a unit has the eight columns 8c .. 8c + 7 (four bytes), from the unit's elements on.
__host__ __device__ inline int fp4_word_offset(int r, int c) { return r * 64 + (((c >> 2) ^ ((r >> 1) & 3)) << 4) + ((c & 3) << 2); }
// ... and the four scales of 64 (groups of 16) or 128 columns, from the unit's start on.
__host__ __device__ inline int fp4_scales_offset(int r, int which) { return which * 512 + (r & 31) * 16 + (r >> 5) * 4; }

// 2^e as a float, e = -127 .. 127.
__device__ __forceinline__ float fp4_two_to(int e) { return __uint_as_float(e > -127 ? (uint32_t)(e + 127) << 23 : 0x00400000u); }

// Exponent of the largest magnitude of a group or row (as bf16 bits without the sign; subnormal numbers have theirs).
__device__ __forceinline__ int fp4_exponent(uint32_t top) {
    const float f = __uint_as_float(top << 16);
    return top >= 0x80u ? (int)(top >> 7) - 127 : ilogbf(f);
}
// The exponent of the power of two in common: the largest scale lands between 170 and 342, of at most 448.  0 for zeros alone.
__device__ __forceinline__ int fp4_common_exponent(uint32_t top) { return top == 0 ? 0 : max(fp4_exponent(top) - 10, -126); }

// Two floats to two elements (x0 in the low half of the byte), ties to the even code, at most 6.
__device__ __forceinline__ uint32_t fp4_pack8(const float (&x)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
    return r;
}
// A byte's two elements, the low half first.
__device__ __forceinline__ float2 fp4_unpack2(uint32_t byte) {
    float2 x;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t.reg .b32 h;\n\t.reg .b16 l, u;\n\tmov.b32 {b0, b1, b2, b3}, %2;\n\tcvt.rn.f16x2.e2m1x2 h, b0;\n\t"
        "mov.b32 {l, u}, h;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}" : "=f"(x.x), "=f"(x.y) : "r"(byte));
    return x;
}
// A positive float to four exponent and three mantissa bits, ties to the even code, and back.
__device__ __forceinline__ uint32_t fp4_scale_code(float s) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(s));
    return r & 0xffu;
}
__device__ __forceinline__ float fp4_scale_value(uint32_t code) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)code));
    float lo;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(lo) : "r"(r));
    return lo;
}

// Eight bf16 numbers (a vector) of a group whose largest magnitude is `top`: their elements, and the group's scale.  `common` is 2^-e of
// the power of two in common (groups of 16).
// All of it is as exact arithmetic would have it.  Groups of 32: multiplying with a power of two is exact.  Groups of 16: the scale is the
// rounding of a quotient, top / 6, that equals the middle between two scales if its fp32 rounding does, because a middle has few bits; an
// element is x / s with x of eight bits and s of at most four, which is either exactly a middle of two elements or at least 2^-10 away
// from one, so that the product with 1 / s, off by less than 2^-20, is brought to the grid of 2^-13 before it is rounded.
template <int kGroup>
__device__ __forceinline__ uint32_t fp4_quantise8(uint4 v, uint32_t top, float common, uint32_t& code) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float x[8];
    if (kGroup == 32) {
        const int e = top == 0 ? -127 : max(fp4_exponent(top) - 2, -127);
        code = (uint32_t)(e + 127);
        const float r = fp4_two_to(-e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]) * r;
            x[2 * i + 1] = bf16_hi(w[i]) * r;
        }
    } else {
        // t / 6 rounded once: a quotient, its exact remainder, and the correction
        const float t = __uint_as_float(top << 16) * common, q = t * (1.f / 6.f);
        code = fp4_scale_code(fmaf(fmaf(-6.f, q, t), 1.f / 6.f, q));
        const float s = fp4_scale_value(code);
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
        r = s > 0.f ? r : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
        if (common > 1e30f) {                                            // the product of the two would leave the range
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= common;
        } else {
            r *= common;
        }
        const unsigned long long rr = ptx::pack_f32x2(r, r), up = ptx::pack_f32x2(1536.f, 1536.f), down = ptx::pack_f32x2(-1536.f, -1536.f);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float2 y = ptx::unpack_f32x2(ptx::add_f32x2(ptx::add_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(x[i], x[i + 1]), rr), up), down));
            x[i] = y.x;
            x[i + 1] = y.y;
        }
    }
    return fp4_pack8(x);
}

// Largest magnitude of a vector of eight, as bits (a number that is not finite has 0x7f80 or more).
__device__ __forceinline__ uint32_t fp4_top8(uint4 v) {
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16);
}
// ... of the group, from its vectors in neighbouring lanes.
template <int kGroup>
__device__ __forceinline__ uint32_t fp4_group_top(uint32_t top) {
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    if (kGroup == 32) top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    return top;
}
// The scales of the eight (groups of 16) or sixteen (32) lanes that hold 64 or 128 columns, as a word in the first of them.
template <int kGroup>
__device__ __forceinline__ uint32_t fp4_gather_codes(uint32_t code) {
    constexpr int step = kGroup / 8;
    uint32_t w = code;
    w |= __shfl_down_sync(0xffffffffu, code, step) << 8;
    w |= __shfl_down_sync(0xffffffffu, code, 2 * step) << 16;
    w |= __shfl_down_sync(0xffffffffu, code, 3 * step) << 24;
    return w;
}

struct Fp4Head {
    const unsigned char* weights;  // behind the header
    const float* weight_factor;    // the power of two that all weights have in common
    const unsigned char* acts;     // [tiles of rows_per_tile rows][blocks] units
    const float* factor;           // [M]: power of two of each row; NaN where the row has values that are not finite
    int M, d, V;
    const float* tau_per_row;
    float tau;
    int* argmax;
    float* entropy;
    float* maxprob;
    unsigned char* exit_mask;
    Control* ctrl;
};

// Few rows (fp4_stream.cu): weights as the M operand.  parts: [CTAs][rows padded] states.  Whole calls at V = 50304, groups of 16, this kernel / the one for
// many rows: 32 rows of 512 11.5 / 19.2 us, of 2560 18.5 / 28.6, 64 rows of 512 15.0 / 20.7, of 1024 15.8 / 22.6, of 2560 21.6 / 29.9, of 8192 50 / 65.  With a
// tile of 128 padded rows, which was built too and not kept: 65 rows of 512 26.0 / 20.8, 100 of 1024 27.1 / 23.0, 128 of 2560 32.5 / 30.5.
constexpr int kFp4StreamRows = 64;
int fp4_stream_padded(int M);                    // rows of a tile of activations
size_t fp4_stream_parts_bytes(int M);
ee_status fp4_stream_launch(const Fp4Head& p, int group, void* parts, int num_sms, int device, cudaStream_t stream);

// Many rows (fp4_gemm.cu): activations as the M operand, 128 rows to a tile.
int fp4_gemm_act_tiles(int M);                   // tiles of activations, the last of them perhaps unused
size_t fp4_gemm_parts_bytes(int M, int V);
ee_status fp4_gemm_launch(const Fp4Head& p, int group, void* parts, int device, cudaStream_t stream);

}  // namespace ee
