// Products of two row-major operands along their rows, D[m][n] = sum_k A[m][k] B[n][k], as a tile of a workgroup: the core of the
// loss over a vocabulary and of the orthogonalised updates.
//
// An operand is rows of 128-byte steps of 16-bit numbers.  One plane (PL = 1): a step is 64 numbers along k.  Two planes (PL = 2): a
// step is 32 numbers along k, the upper parts first, then what they leave; the product takes upper x upper and the two mixed ones, and
// leaves out lower x lower (2^-22 of the product for binary16 planes).
#pragma once
#include "monarch_mfma_common.h"

namespace monarch {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

struct NtOperand {
    const void* base;    // 16-byte aligned
    int64_t rows;        // rows from here on read as zeros
    uint32_t row_bytes;  // a multiple of 16; a tile's rows stay below 2^31 bytes
};

// A workgroup's BM x BN tile, a wave's WM x WN part of it.
template <int BM_, int BN_, int WM_, int WN_, int PL_, bool F16_>
struct NtTile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, PL = PL_;
    static constexpr bool F16 = F16_;
    static constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = 64 * WAVES;
    static constexpr int TI = WM / 16, TJ = WN / 16;
    static constexpr int BUFFER = (BM + BN) * 128, LDS_BYTES = 2 * BUFFER;
    static constexpr int ASK_A = BM / 8 / WAVES, ASK_B = BN / 8 / WAVES;  // requests of a wave per step, 8 rows each
    static_assert(ASK_A * 8 * WAVES == BM && ASK_B * 8 * WAVES == BN, "whole requests");
    static __device__ __forceinline__ int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
    static __device__ __forceinline__ int row0() { return wave() / (BN / WN) * WM; }  // of the wave's part
    static __device__ __forceinline__ int col0() { return wave() % (BN / WN) * WN; }
};

template <bool F16>
__device__ __forceinline__ f32x4 nt_mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return mfma16(as_bf16x8(a), as_bf16x8(b), c);
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
// Double buffer: while a step's products run, the next one's 128-byte rows come straight into the other half of LDS.  16-byte piece u
// of row r lies in place u ^ (r % 8), so that the 16 rows of a fragment fall on different banks.
template <typename C>
__device__ __forceinline__ void nt_product(const NtOperand& A, int64_t a0, const NtOperand& B, int64_t b0, int step0, int steps,
                                           unsigned char* lds, f32x4 (&acc)[C::TI][C::TJ])
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
    if (steps > 0) ask(step0, 0);
    for (int s = 0; s < steps; ++s) {
        const int buffer = s & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + 1 < steps) ask(step0 + s + 1, buffer ^ 1);
        const unsigned char *pa = fa + buffer * C::BUFFER, *pb = fb + buffer * C::BUFFER;
        u32x4 b[2][C::TJ];
#pragma unroll
        for (int j = 0; j < C::TJ; ++j) {
            b[0][j] = lds128(pb + j * 2048 + at0);
            b[1][j] = lds128(pb + j * 2048 + at1);
        }
#pragma unroll
        for (int i = 0; i < C::TI; ++i) {
            const u32x4 a0 = lds128(pa + i * 2048 + at0), a1 = lds128(pa + i * 2048 + at1);
#pragma unroll
            for (int j = 0; j < C::TJ; ++j) {
                acc[i][j] = nt_mfma<C::F16>(a0, b[0][j], acc[i][j]);
                if constexpr (C::PL == 1) {
                    acc[i][j] = nt_mfma<C::F16>(a1, b[1][j], acc[i][j]);
                } else {
                    acc[i][j] = nt_mfma<C::F16>(a0, b[1][j], acc[i][j]);
                    acc[i][j] = nt_mfma<C::F16>(a1, b[0][j], acc[i][j]);
                }
            }
        }
    }
#endif
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
