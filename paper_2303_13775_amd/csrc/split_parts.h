// A float as three bfloat16 parts, and the products of 16 k on the matrix units (included inside anonymous namespaces, after
// gemm_common.h).  What the parts carry, and what is summed of their products: gemm_split.h.
#pragma once

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int SPLIT_MIN_K = 3;          // shorter contractions are formed with fp32 MFMAs
constexpr float SPLIT_SCALE = 0x1p16f, SPLIT_UNSCALE = 0x1p-32f;        // of an operand, of a product of two

__device__ __forceinline__ uint32_t cvt2bf(float a, float b) {      // round to nearest even, a in the low half
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}
// two values -> one word (two bfloat16) of each of the three parts
__device__ __forceinline__ void split2(float a, float b, uint32_t &p1, uint32_t &p2, uint32_t &p3) {
    p1 = cvt2bf(a, b);
    a -= __uint_as_float(p1 << 16); b -= __uint_as_float(p1 & 0xFFFF0000u);
    p2 = cvt2bf(a, b);
    a -= __uint_as_float(p2 << 16); b -= __uint_as_float(p2 & 0xFFFF0000u);
    p3 = cvt2bf(a, b);
}
__device__ __forceinline__ void split8(const float (&v)[8], uint4 (&p)[3]) {
    split2(v[0], v[1], p[0].x, p[1].x, p[2].x);
    split2(v[2], v[3], p[0].y, p[1].y, p[2].y);
    split2(v[4], v[5], p[0].z, p[1].z, p[2].z);
    split2(v[6], v[7], p[0].w, p[1].w, p[2].w);
}
__device__ __forceinline__ floatx16 mfma_bf(const uint4 &a, const uint4 &b, const floatx16 &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 zero16() {
    floatx16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
__device__ __forceinline__ bool finite16(const floatx16 &v) {
    bool ok = true;
#pragma unroll
    for (int r = 0; r < 16; ++r) ok = ok && fabsf(v[r]) < INFINITY;
    return ok;
}
// contraction index j of granule g of a tile of 32 k (see the fragments in gemm_split.h)
__device__ __forceinline__ int granule_k(int g, int j) { return 4 * g + j + (j < 4 ? 0 : 12); }

// The products of k_begin .. k_end - 1 with fp32 MFMAs, sums of 16 k added up (a single chain of 64 k rounded more
// often than the fp32 tiles whose waves each took a part of the contraction: 2.4 units of 2^-24 against 1.4).
template <class GetA, class GetB>
__device__ __forceinline__ floatx16 exact_sum(int k_begin, int k_end, int half, const GetA &get_a, const GetB &get_b) {
    floatx16 sum = zero16();
#pragma unroll 1
    for (int k0 = k_begin; k0 < k_end; k0 += 16) {
        floatx16 part = zero16();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int k = k0 + 8 * half + q;
            part = __builtin_amdgcn_mfma_f32_32x32x2f32(get_a(k), get_b(k), part, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[r] += part[r];
    }
    return sum;
}
