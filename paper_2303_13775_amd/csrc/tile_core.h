// The contraction of large tiles of half-precision products (included inside anonymous namespaces).  A stage of the contraction is 128 bytes of every row of either operand; two stages lie in LDS.
// Operands go from memory straight into LDS, no register holds them on the way, and a wave reads the fragments of one step while
// the matrix unit works on those of the step in front:
//     step s of stage t:  read the fragments of step s + 1; matrix instructions of step s
//     its last step:      wait for stage t + 1, read its first fragments, fetch stage t + 2 into the place of stage t, and then the
//                         matrix instructions
// so one barrier a stage has the matrix instructions of the other wave on the SIMD to hide behind, and a fetch a whole stage's.
#pragma once

typedef float floatx16_t __attribute__((ext_vector_type(16)));
typedef uint32_t core_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t core_u32x4 __attribute__((ext_vector_type(4)));
typedef short core_s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int core_wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// 64 lanes fetch 16 bytes each into 1 KB of LDS side by side.  (Not the compiler's built-in function: it has every transposed read of
// LDS wait for all fetches on their way, whatever place they write, which left none of them in flight behind the matrix instructions.
// Nothing here waits for a fetch but core_landed.  The place in LDS is an operand in m0, which the instruction reads one wait state after
// it is set: the compiler sets it, and knows what else it keeps there.)
__device__ __forceinline__ void core_fetch(const void *from, core_u32x4 *to) {
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)to);
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(at), "v"(from) : "memory");
}

// Operand rows of 128 bytes a stage, eight granules of 16 each.  Granule p of row r of LDS holds granule p ^ (r / 2) % 8: sixteen rows of
// one granule column lie in sixteen groups of banks.
__device__ __forceinline__ int along_turn(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int along_at(int row, int g) { return row * 8 + (g ^ along_turn(row)); }
// what lane `lane` of the instruction that fetches rows 8 x .. 8 x + 7 asks for: its row among them, its granule
__device__ __forceinline__ int along_row(int lane) { return lane >> 3; }
__device__ __forceinline__ int along_granule(int x, int lane) { return (lane & 7) ^ along_turn((8 * x & 8) + (lane >> 3)); }

// Where a wave reads its rows' fragments from: granule 2 h + lane / 32 of row `first` + lane % 32 (first: a multiple of 32, `from`: where
// the operand's rows start).  The other steps' and the rows further on lie an exclusive or and a constant away.
__device__ __forceinline__ int along_base(int from, int first) {
    const int lane = threadIdx.x & 63;
    return from + first * 8 + along_at(lane & 31, lane >> 5);
}
__device__ __forceinline__ core_u32x4 along_fragment(const core_u32x4 *lds, int base, int h, int block) { return lds[(base ^ (2 * h)) + 256 * block]; }

// Operand with the contraction across its rows, read transposed: a row holds ROW granules.  Granule p of row r holds granule
// p ^ 4 (r % 4): the four rows that 32 lanes read 64 bytes of lie in different banks.
// Fragments are eight rows 16 h + 8 (lane / 32) .. of 32 columns, one a lane, whose values start at granule `first`.  Of sixteen lanes each
// supplies four columns of one of four rows and gets one column of all four.
template <int ROW> __device__ __forceinline__ int across_base(int from, int first) {       // in halves of a granule
    const int lane = threadIdx.x & 63, row = 8 * (lane >> 5) + ((lane & 15) >> 2);
    return 2 * (from + row * ROW + ((first + 2 * (lane >> 4 & 1) + (lane >> 1 & 1)) ^ (4 * (row & 3)))) + (lane & 1);
}
// `further`: granules that `first` lies further on, bits that it has not set
template <int ROW>
__device__ __forceinline__ core_u32x4 across_fragment(const core_u32x4 *lds, int base, int h, int further) {
    typedef __attribute__((address_space(3))) core_s16x4 *P;
    const auto at = [&](int row) { return (P)((__attribute__((address_space(3))) const core_u32x2 *)lds + (base ^ (2 * further)) + 2 * ROW * row); };
    const core_u32x2 a = __builtin_bit_cast(core_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(16 * h)));
    const core_u32x2 b = __builtin_bit_cast(core_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(16 * h + 4)));
    return core_u32x4{a[0], a[1], b[0], b[1]};
}

// STEPS steps a stage.  fetch(t, lds): stage t of both operands into lds; Frag read(lds, s); multiply(frag).
// Waits until this wave's fetches have landed, and for the other waves' to have.
__device__ __forceinline__ void core_landed() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}
template <int STEPS, class Frag, int WORDS, class Fetch, class Read, class Multiply>
__device__ __forceinline__ void core_contract(int stages, core_u32x4 (&lds)[2][WORDS], const Fetch &fetch, const Read &read, const Multiply &multiply) {
    static_assert(STEPS % 2 == 0, "the first step of a stage finds its fragments in the first place");
    Frag f[2];
    fetch(0, lds[0]);
    core_landed();
    if (stages > 1) fetch(1, lds[1]);
    read(f[0], lds[0], 0);
    // (the last stage by itself: where its branch met the others', the fragments just asked for were waited for)
    for (int t = 0; t + 1 < stages; ++t) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s + 1 < STEPS) {
                read(f[(s + 1) & 1], lds[t & 1], s + 1);
            } else {
                core_landed();
                read(f[0], lds[(t + 1) & 1], 0);
                if (t + 2 < stages) fetch(t + 2, lds[t & 1]);
            }
            multiply(f[s & 1]);
        }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (s + 1 < STEPS) read(f[(s + 1) & 1], lds[(stages - 1) & 1], s + 1);
        multiply(f[s & 1]);
    }
}
// The same for a wave that has nothing to form: its share of the fetches, and the barriers.
template <int WORDS, class Fetch>
__device__ __forceinline__ void core_idle(int stages, core_u32x4 (&lds)[2][WORDS], const Fetch &fetch) {
    fetch(0, lds[0]);
    core_landed();
    if (stages > 1) fetch(1, lds[1]);
    for (int t = 0; t + 1 < stages; ++t) {
        core_landed();
        if (t + 2 < stages) fetch(t + 2, lds[t & 1]);
    }
}
