// Products D[m][n] = sum_k A[m][k] B[n][k] as a tile of a workgroup: the core of the loss over a vocabulary and of the orthogonalised updates.
//
// An operand lies in memory along k (rows m, a row's numbers along k) or across it (rows k, a row's numbers along m), as rows of 128-byte pieces,
// and comes as steps of 64 or 32 numbers of k.  What 128 bytes hold goes by the kind:
//   kBf16, kF16     64 numbers (a step: 64 of k)
//   kF16x2          32 numbers in two binary16 planes, the upper parts first, then what they leave (a step: 32 of k); the product takes
//                   upper x upper and the two mixed ones, and leaves out lower x lower (2^-22 of the product)
//   kF32            32 fp32 numbers along k (a step: 32 of k), on the fp32 matrix instruction (a sixteenth of the bf16 rate)
#pragma once
#include <type_traits>

#include "monarch_lds_tr.h"

namespace monarch {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

struct NtOperand {
    const void* base;    // 16-byte aligned
    int64_t rows;        // rows from here on read as zeros
    uint32_t row_bytes;  // a multiple of 16; the rows of a tile, or of a step, stay below 2^31 bytes
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

#ifdef __HIP_DEVICE_COMPILE__  // (buffer descriptors are no type of the host's)
// `rows` rows (less where the operand ends) from `row`, `skip` bytes into it
__device__ __forceinline__ auto nt_rsrc(const NtOperand& o, int64_t row, int rows_of_tile, uint32_t skip)
{
    int64_t rows = o.rows - row;
    rows = rows < 0 ? 0 : rows > rows_of_tile ? rows_of_tile : rows;
    const uint32_t bytes = (uint32_t)rows * o.row_bytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((const char*)o.base) + row * (int64_t)o.row_bytes + skip, 0,
                                             (int)(bytes > skip ? bytes - skip : 0), 0x00020000);
}

// One operand of a tile: SIDE (BM or BN) rows of it along k, or SIDE columns of it across k.  In LDS a step is SIDE x 128 bytes.
//   along k: 128-byte rows, 16-byte piece u of row r in place u ^ (r % 8), so that the 16 rows of a fragment fall on different banks;
//   across k: rows of one k, 32-byte piece u in place u ^ (the row's key): a transposing read of 32 lanes touches one piece each of rows
//   8g .. 8g+3 and 8g+8 .. 8g+11, which have different keys and so fall on different banks.
template <typename C, int SIDE, int ASKS, bool ACROSS>
struct NtSide {
    static constexpr int ROW = ACROSS ? SIDE * 2 * C::PL : 128, K_ROWS = 64 / C::PL;
    static_assert(!ACROSS || ROW >= 256, "pieces for eight keys");
    const NtOperand& o;
    int64_t first;  // row (column) of the tile
    uint32_t at[ASKS];
    // (a descriptor for the whole tile, or made anew for every step's rows)
    __device__ __forceinline__ NtSide(const NtOperand& operand, int64_t tile0, int wave, int lane) : o(operand), first(tile0)
    {
#pragma unroll
        for (int i = 0; i < ASKS; ++i) {
            if constexpr (ACROSS) {
                const uint32_t p = (wave + i * C::WAVES) * 1024 + lane * 16, row = p / ROW, in = p % ROW, key = (row & 3) | (row >> 3 & 1) << 2;
                at[i] = row * o.row_bytes + (in ^ key << 5);
            } else {
                at[i] = ((wave + i * C::WAVES) * 8 + (lane >> 3)) * o.row_bytes + 16 * ((lane & 7) ^ (lane >> 3));
            }
        }
    }
    template <typename P>
    __device__ __forceinline__ void ask(int step, P to) const  // to: of the wave's first request
    {
        const auto r = ACROSS ? nt_rsrc(o, (int64_t)step * K_ROWS, K_ROWS, (uint32_t)(first * 2 * C::PL)) : nt_rsrc(o, first, SIDE, 0);
#pragma unroll
        for (int i = 0; i < ASKS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + i * C::WAVES * 1024), 16, at[i],
                                                     ACROSS ? 0 : step * 128, 0, 0);
    }
};

// The fragment of 16 columns from `col` on of an operand across k, on its way from LDS (its waits are the caller's): half 0 and 1 are the step's two
// halves of k, or the two planes.  `lane_at`: where the lane's first row lies, with its key.
template <typename C, int ROW>
__device__ __forceinline__ void nt_read_across(uint32_t lane_at, int col, Frag (&f)[2])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t piece = C::PL == 1 ? col >> 4 : (uint32_t)((col >> 5) * 4 + 2 * h + (col >> 4 & 1));
        const uint32_t at = (lane_at ^ (piece & 7) << 5) + (piece >> 3) * 256;
        if (C::PL == 1 && h) {
            f[h].lo = lds_tr16<32 * ROW>(at);
            f[h].hi = lds_tr16<36 * ROW>(at);
        } else {
            f[h].lo = lds_tr16<0>(at);
            f[h].hi = lds_tr16<4 * ROW>(at);
        }
    }
}
__device__ __forceinline__ u32x4 nt_whole(const Frag& f) { return u32x4{f.lo[0], f.lo[1], f.hi[0], f.hi[1]}; }
#endif

// acc[i][j][e] = D[a0 + row0() + 16 i + 4 (lane / 16) + e][b0 + col0() + 16 j + lane % 16] over `steps` steps from `step0`.
// The next RING - 1 steps come straight into LDS while a step's products run; one barrier a step.  KA, KB: A, B lie across k.  TAIL (both along k): only
// the first `tail` of the eight 16-byte pieces of the last step count (the rows end there, and what follows is not theirs).
template <typename C, bool TAIL = false, bool KA = false, bool KB = false>
__device__ __forceinline__ void nt_product(const NtOperand& A, int64_t a0, const NtOperand& B, int64_t b0, int step0, int steps,
                                           unsigned char* lds, f32x4 (&acc)[C::TI][C::TJ], int tail = 8)
{
#pragma unroll
    for (int i = 0; i < C::TI; ++i)
#pragma unroll
        for (int j = 0; j < C::TJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#ifdef __HIP_DEVICE_COMPILE__
    const int wave = C::wave(), lane = threadIdx.x & 63;
    using SideA = NtSide<C, C::BM, C::ASK_A, KA>;
    using SideB = NtSide<C, C::BN, C::ASK_B, KB>;
    const SideA side_a(A, a0, wave, lane);
    const SideB side_b(B, b0, wave, lane);
    auto to = (__attribute__((address_space(3))) unsigned char*)lds + wave * 1024;
    auto ask = [&](int step, int buffer) {
        side_a.ask(step, to + buffer * C::BUFFER);
        side_b.ask(step, to + buffer * C::BUFFER + C::BM * 128);
    };
    const int r16 = lane & 15, at0 = 16 * ((lane >> 4) ^ (lane & 7)), at1 = at0 ^ 64;
    const unsigned char* fa = lds + (C::row0() + r16) * 128;
    const unsigned char* fb = lds + C::BM * 128 + (C::col0() + r16) * 128;
    // across k: the lane's row among 8g .. 8g+3, its key, its four columns
    const uint32_t row_k = 8 * (lane >> 4) + (r16 >> 2), in_k = ((row_k & 3) | (row_k >> 3 & 1) << 2) << 5 | 8 * (lane & 3);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    const uint32_t ka = lds0 + row_k * SideA::ROW + in_k, kb = lds0 + C::BM * 128 + row_k * SideB::ROW + in_k;
    auto products = [&](auto cut, int buffer) {
        const unsigned char *pa = fa + buffer * C::BUFFER, *pb = fb + buffer * C::BUFFER;
        const bool in0 = lane >> 4 < tail, in1 = 4 + (lane >> 4) < tail;
        auto half = [&](const unsigned char* p, bool in) {
            u32x4 v = lds128(p);
            if constexpr (decltype(cut)::value)
                if (!in) v = u32x4{0, 0, 0, 0};
            return v;
        };
        u32x4 b[2][C::TJ];
        if constexpr (!KB) {
#pragma unroll
            for (int j = 0; j < C::TJ; ++j) {
                b[0][j] = half(pb + j * 2048 + at0, in0);
                b[1][j] = half(pb + j * 2048 + at1, in1);
            }
        }
        Frag a[2][2], bk[KB ? C::TJ : 1][2];
        if constexpr (KB) {
#pragma unroll
            for (int j = 0; j < C::TJ; ++j) nt_read_across<C, SideB::ROW>(kb + buffer * C::BUFFER, C::col0() + 16 * j, bk[j]);
        }
        if constexpr (KA) {
            nt_read_across<C, SideA::ROW>(ka + buffer * C::BUFFER, C::row0(), a[0]);
            lgkm_wait(a[0]);
        }
        if constexpr (KB) {
#pragma unroll
            for (int j = 0; j < C::TJ; ++j) {
                lgkm_wait(bk[j]);
                b[0][j] = nt_whole(bk[j][0]);
                b[1][j] = nt_whole(bk[j][1]);
            }
        }
        if constexpr (KA) {
#pragma unroll
            for (int i = 0; i < C::TI; ++i) {
                // (the next fragment travels during this one's products)
                if (i + 1 < C::TI) nt_read_across<C, SideA::ROW>(ka + buffer * C::BUFFER, C::row0() + 16 * (i + 1), a[(i + 1) & 1]);
#pragma unroll
                for (int j = 0; j < C::TJ; ++j)
                    acc[i][j] = nt_step<C::KIND>(nt_whole(a[i & 1][0]), nt_whole(a[i & 1][1]), b[0][j], b[1][j], acc[i][j]);
                if (i + 1 < C::TI) lgkm_wait(a[(i + 1) & 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < C::TI; ++i) {
                const u32x4 u = half(pa + i * 2048 + at0, in0), v = half(pa + i * 2048 + at1, in1);
#pragma unroll
                for (int j = 0; j < C::TJ; ++j) acc[i][j] = nt_step<C::KIND>(u, v, b[0][j], b[1][j], acc[i][j]);
            }
        }
    };
    constexpr int PENDING = C::ASK_A + C::ASK_B;
    for (int s = 0; s < C::RING - 1 && s < steps; ++s) ask(step0 + s, s);
    int buffer = 0;
    for (int s = 0; s < steps; ++s) {
        // step s has landed once only what was asked for after it is outstanding
        if (C::RING == 4 && s + 2 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * PENDING) : "memory");
        else if (C::RING >= 3 && s + 1 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PENDING) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();  // ... for every wave, and nobody reads step s - 1 any more
        asm volatile("" ::: "memory");
        if (s + C::RING - 1 < steps) ask(step0 + s + C::RING - 1, buffer ? buffer - 1 : C::RING - 1);
        if (TAIL && s + 1 == steps && tail < 8) products(std::true_type{}, buffer);
        else products(std::false_type{}, buffer);
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
