// Products of two row-major operands along their rows, D[m][n] = sum_k A[m][k] B[n][k], as a tile of a workgroup: the core of the
// loss over a vocabulary and of the orthogonalised updates.
//
// An operand is rows of 128-byte steps.  What a step holds goes by the kind:
//   kBf16, kF16     64 numbers along k
//   kF16x2          32 numbers along k in two binary16 planes, the upper parts first, then what they leave; the product takes upper x
//                   upper and the two mixed ones, and leaves out lower x lower (2^-22 of the product)
//   kF32            32 fp32 numbers along k, on the fp32 matrix instruction (a sixteenth of the bf16 rate)
#pragma once
#include <type_traits>

#include "monarch_mfma_common.h"

namespace monarch {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

struct NtOperand {
    const void* base;    // 16-byte aligned
    int64_t rows;        // rows from here on read as zeros
    uint32_t row_bytes;  // a multiple of 16; a tile's rows stay below 2^31 bytes
};

enum NtKind { kBf16, kF16, kF16x2, kF32 };

// A workgroup's BM x BN tile, a wave's WM x WN part of it.
template <int BM_, int BN_, int WM_, int WN_, NtKind KIND_, int RING_ = 2>
struct NtTile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, RING = RING_;  // RING: steps in LDS
    static constexpr NtKind KIND = KIND_;
    static constexpr int PL = KIND == kF16x2 ? 2 : 1;  // planes
    static constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = 64 * WAVES;
    static constexpr int TI = WM / 16, TJ = WN / 16;
    static constexpr int BUFFER = (BM + BN) * 128, LDS_BYTES = RING * BUFFER;
    static constexpr int ASK_A = BM / 8 / WAVES, ASK_B = BN / 8 / WAVES;  // requests of a wave per step, 8 rows each
    static_assert(RING >= 2 && RING <= 4, "ring");
    static_assert(ASK_A * 8 * WAVES == BM && ASK_B * 8 * WAVES == BN, "whole requests");
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
    static __device__ __forceinline__ int row0() { return wave() / (BN / WN) * WM; }  // of the wave's part
    static __device__ __forceinline__ int col0() { return wave() % (BN / WN) * WN; }
};

__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// c += what a step's two halves of the operands contribute
template <NtKind KIND>
__device__ __forceinline__ f32x4 nt_step(u32x4 a0, u32x4 a1, u32x4 b0, u32x4 b1, f32x4 c)
{
    if constexpr (KIND == kBf16) {
        c = mfma16(as_bf16x8(a0), as_bf16x8(b0), c);
        return mfma16(as_bf16x8(a1), as_bf16x8(b1), c);
    } else if constexpr (KIND == kF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a0[e]), __uint_as_float(b0[e]), c, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a1[e]), __uint_as_float(b1[e]), c, 0, 0, 0);
        return c;
    } else {
        const f16x8 p0 = __builtin_bit_cast(f16x8, a0), p1 = __builtin_bit_cast(f16x8, a1), q0 = __builtin_bit_cast(f16x8, b0), q1 = __builtin_bit_cast(f16x8, b1);
        c = mfma16(p0, q0, c);
        if constexpr (KIND == kF16) return mfma16(p1, q1, c);
        c = mfma16(p0, q1, c);
        return mfma16(p1, q0, c);
    }
}

#ifdef __HIP_DEVICE_COMPILE__
__device__ __forceinline__ auto nt_rsrc(const NtOperand& o, int64_t row, int rows_of_tile)
{
    int64_t rows = o.rows - row;
    rows = rows < 0 ? 0 : rows > rows_of_tile ? rows_of_tile : rows;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((const char*)o.base) + row * (int64_t)o.row_bytes, 0,
                                             (int)(rows * o.row_bytes), 0x00020000);
}
#endif

// acc[i][j][e] = D[a0 + row0() + 16 i + 4 (lane / 16) + e][b0 + col0() + 16 j + lane % 16] over `steps` steps from `step0`.
// The 128-byte rows of the next RING - 1 steps come straight into LDS while a step's products run; one barrier a step.  16-byte piece u
// of row r lies in place u ^ (r % 8), so that the 16 rows of a fragment fall on different banks.  TAIL: only the first `tail` of the eight
// pieces of the last step count (the rows end there, and what follows is not theirs).
template <typename C, bool TAIL = false>
__device__ __forceinline__ void nt_product(const NtOperand& A, int64_t a0, const NtOperand& B, int64_t b0, int step0, int steps,
                                           unsigned char* lds, f32x4 (&acc)[C::TI][C::TJ], int tail = 8)
{
#pragma unroll
    for (int i = 0; i < C::TI; ++i)
#pragma unroll
        for (int j = 0; j < C::TJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#ifdef __HIP_DEVICE_COMPILE__  // (buffer descriptors are no type of the host's)
    const int wave = C::wave(), lane = threadIdx.x & 63;
    const auto ra = nt_rsrc(A, a0, C::BM), rb = nt_rsrc(B, b0, C::BN);
    const uint32_t piece = 16 * ((lane & 7) ^ (lane >> 3)), row = wave * 8 + (lane >> 3);
    uint32_t va[C::ASK_A], vb[C::ASK_B];
#pragma unroll
    for (int i = 0; i < C::ASK_A; ++i) va[i] = (row + i * 8 * C::WAVES) * A.row_bytes + piece;
#pragma unroll
    for (int i = 0; i < C::ASK_B; ++i) vb[i] = (row + i * 8 * C::WAVES) * B.row_bytes + piece;
    auto to = (__attribute__((address_space(3))) unsigned char*)lds + wave * 1024;
    auto ask = [&](int step, int buffer) {
#pragma unroll
        for (int i = 0; i < C::ASK_A; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (__attribute__((address_space(3))) void*)(to + buffer * C::BUFFER + i * C::WAVES * 1024), 16,
                                                     va[i], step * 128, 0, 0);
#pragma unroll
        for (int i = 0; i < C::ASK_B; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (__attribute__((address_space(3))) void*)(to + buffer * C::BUFFER + C::BM * 128 + i * C::WAVES * 1024), 16,
                                                     vb[i], step * 128, 0, 0);
    };
    const int r16 = lane & 15, at0 = 16 * ((lane >> 4) ^ (lane & 7)), at1 = at0 ^ 64;
    const unsigned char* fa = lds + (C::row0() + r16) * 128;
    const unsigned char* fb = lds + C::BM * 128 + (C::col0() + r16) * 128;
    auto products = [&](auto cut, const unsigned char* pa, const unsigned char* pb) {
        const bool in0 = lane >> 4 < tail, in1 = 4 + (lane >> 4) < tail;
        auto half = [&](const unsigned char* p, bool in) {
            u32x4 v = lds128(p);
            if constexpr (decltype(cut)::value)
                if (!in) v = u32x4{0, 0, 0, 0};
            return v;
        };
        u32x4 b[2][C::TJ];
#pragma unroll
        for (int j = 0; j < C::TJ; ++j) {
            b[0][j] = half(pb + j * 2048 + at0, in0);
            b[1][j] = half(pb + j * 2048 + at1, in1);
        }
#pragma unroll
        for (int i = 0; i < C::TI; ++i) {
            const u32x4 a0 = half(pa + i * 2048 + at0, in0), a1 = half(pa + i * 2048 + at1, in1);
#pragma unroll
            for (int j = 0; j < C::TJ; ++j) acc[i][j] = nt_step<C::KIND>(a0, a1, b[0][j], b[1][j], acc[i][j]);
        }
    };
    constexpr int ASKS = C::ASK_A + C::ASK_B;
    for (int s = 0; s < C::RING - 1 && s < steps; ++s) ask(step0 + s, s);
    int buffer = 0;
    for (int s = 0; s < steps; ++s) {
        // step s has landed once only what was asked for after it is outstanding
        if (C::RING == 4 && s + 2 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * ASKS) : "memory");
        else if (C::RING >= 3 && s + 1 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(ASKS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // ... for every wave, and nobody reads step s - 1 any more
        asm volatile("" ::: "memory");
        if (s + C::RING - 1 < steps) ask(step0 + s + C::RING - 1, buffer ? buffer - 1 : C::RING - 1);
        const unsigned char *pa = fa + buffer * C::BUFFER, *pb = fb + buffer * C::BUFFER;
        if (TAIL && s + 1 == steps && tail < 8) products(std::true_type{}, pa, pb);
        else products(std::false_type{}, pa, pb);
        buffer = buffer + 1 == C::RING ? 0 : buffer + 1;
    }
#endif
}

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2_t)); }
// Two numbers in binary16 (packed, rounded to nearest), and what that leaves of them.
__device__ __forceinline__ uint32_t take_f16x2(float& a, float& b)
{
    const uint32_t u = pack_f16x2(a, b);
    const f16x2_t h = __builtin_bit_cast(f16x2_t, u);
    a = fmaf((float)h[0], -1.f, a);  // (one instruction, exact)
    b = fmaf((float)h[1], -1.f, b);
    return u;
}
// four numbers as two planes
struct TwoPlanes {
    u32x2 p[2];
};
__device__ __forceinline__ TwoPlanes split_planes(f32x4 v)
{
    float a = v[0], b = v[1], c = v[2], d = v[3];
    TwoPlanes r;
    r.p[0] = u32x2{take_f16x2(a, b), take_f16x2(c, d)};
    r.p[1] = u32x2{pack_f16x2(a, b), pack_f16x2(c, d)};
    return r;
}

// Among four lanes (4q .. 4q + 3) with four 16-bit numbers each: lane i gets number i of all four.
__device__ __forceinline__ u32x2 change_places(u32x2 v)
{
    const int lane = threadIdx.x;
    const uint32_t a = v[0], b = v[1];
    const uint32_t oa = __builtin_amdgcn_mov_dpp((int)a, 0xB1, 0xF, 0xF, true), ob = __builtin_amdgcn_mov_dpp((int)b, 0xB1, 0xF, 0xF, true);
    const uint32_t c = lane & 1 ? pick_hi16(oa, a) : pick_lo16(a, oa), d = lane & 1 ? pick_hi16(ob, b) : pick_lo16(b, ob);
    const uint32_t oc = __builtin_amdgcn_mov_dpp((int)c, 0x4E, 0xF, 0xF, true), od = __builtin_amdgcn_mov_dpp((int)d, 0x4E, 0xF, 0xF, true);
    return lane & 2 ? u32x2{od, d} : u32x2{c, oc};
}

// Tile of a workgroup: the eight XCDs take workgroups in turn, and each gets a run of tiles that lie together (groups of 8 tiles along m, n
// inside), so that what they read is shared in its L2.  False: no tile.
__device__ __forceinline__ bool nt_place(int id, int tiles_m, int tiles_n, int& tm, int& tn)
{
    const int tiles = tiles_m * tiles_n, each = (tiles + 7) >> 3, t = (id & 7) * each + (id >> 3);
    if ((id >> 3) >= each || t >= tiles) return false;
    constexpr int G = 8;
    const int group = t / (G * tiles_n), in = t - group * G * tiles_n, high = tiles_m - group * G < G ? tiles_m - group * G : G;
    tm = group * G + in % high;
    tn = in / high;
    return true;
}
inline int nt_grid(int tiles_m, int tiles_n) { return (tiles_m * tiles_n + 7) / 8 * 8; }

}  // namespace monarch
