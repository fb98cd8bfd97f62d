// Microscaled codes: blocks of 32 columns of a row share one power of two 2^e, kept as the byte e + 127; the elements are E4M3
// (8 bits, checkpoints) or E2M1 (4 bits, two to a byte, the even column in the low half).
//
//   e = floor(log2 amax) - emax, one more where amax's significand is above 1.75;  -127 at the least (and for a block of zeros)
//   code = round_to_nearest_even(x * 2^-e), beyond the largest value that value
//
// emax is 8 for E4M3 and 2 for E2M1.  1.75 * 2^8 = 448 is the end of E4M3, so nothing saturates there.  1.75 * 2^2 = 7 is the middle
// between E2M1's largest value 6 and the next power of two: letting the block's largest value lose up to a seventh leaves the others a
// finer step.  Of the thresholds 1, 1.25 .. 2 it has the least error: root mean square 11.2 % on normal data (1.5, where nothing
// saturates: 11.6 %, always floor: 11.5 %), 16.1 % with one channel in 33 twenty times larger (17.0, 16.9 %).
// E4M3 for the checkpoints and not integers: beside a channel twenty times larger, in its block of 32, integers leave a step of half a
// standard deviation to the others, E4M3 2.6 % of each value.
// A block that holds an infinity or a NaN has the byte 255 and stands for NaN throughout.  Finite values stay finite: in blocks of the
// largest exponent (masks of the type's lowest value are there), codes that would stand for 2^128 are the ones below.
#pragma once
#include "falqon_internal.h"
#include "quantize_common.h"

namespace falqon {
namespace {

constexpr int MX_BLOCK = 32;
constexpr int MX_E4M3_EMAX = 8, MX_E2M1_EMAX = 2;

template <int CTRL>
__device__ __forceinline__ float dpp_move(float x, std::integral_constant<int, CTRL>)
{
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// Largest bit pattern without its sign: the maximum of absolute values, in which a NaN is above an infinity and that above the rest.
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// over the 32 / E lanes that hold a block (E = 8: a quad; E = 4: half a row of 16)
template <int E>
__device__ __forceinline__ uint32_t block_max_bits(uint32_t v)
{
    v = umax(v, __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true));
    v = umax(v, __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true));
    if (E == 4) v = umax(v, __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true));
    return v;
}

// largest absolute value in a lane's 16 bytes, as fp32 bits: fp32, or bf16 two at a time as 16-bit integers
__device__ __forceinline__ uint32_t abs_max_bits(v4u w, const float*)
{
    return umax(umax(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), umax(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
}
__device__ __forceinline__ uint32_t abs_max_bits(v4u w, const uint16_t*)
{
    typedef uint16_t v2h __attribute__((ext_vector_type(2)));
    v2h m = __builtin_bit_cast(v2h, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(v2h, w[i] & 0x7fff7fffu));
    return static_cast<uint32_t>(m[0] > m[1] ? m[0] : m[1]) << 16;
}

// the byte of a block whose largest absolute value has these bits
template <int EMAX>
__device__ __forceinline__ int mx_exponent(uint32_t amax_bits)
{
    int e = static_cast<int>(amax_bits >> 23) - EMAX + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < 0 ? 0 : e;
    return amax_bits >= 0x7f800000u ? 255 : e;
}

// 2^-e of the byte e + 127 <= 247 (what mx_exponent gives for finite blocks and E4M3; 253 for E2M1): at least 2^-126
__device__ __forceinline__ float mx_down(int byte) { return __uint_as_float(static_cast<uint32_t>(254 - byte) << 23); }
// 2^e; 2^-127 is subnormal, 255 NaN
__device__ __forceinline__ float mx_up(int byte)
{
    const float v = __uint_as_float(byte == 0 ? 0x400000u : static_cast<uint32_t>(byte) << 23);
    return byte == 255 ? __uint_as_float(0x7fc00000u) : v;
}

// E4M3 codes of four values under a block's factor; `byte` 255: codes of NaN
__device__ __forceinline__ uint32_t mx8_codes4(float a, float b, float c, float d, float down, int byte)
{
    const float end = byte == 247 ? 240.0f : 448.0f;                  // 247: 2^120, where 256 is out of range
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(a * down, -end, end), __builtin_amdgcn_fmed3f(b * down, -end, end), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(c * down, -end, end), __builtin_amdgcn_fmed3f(d * down, -end, end), w, true);
    return byte == 255 ? 0x7f7f7f7fu : static_cast<uint32_t>(w);
}

typedef float v2f __attribute__((ext_vector_type(2)));
// four codes -> values under a block's factor
__device__ __forceinline__ void mx8_values4(uint32_t w, float up, float (&f)[4])
{
    const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    f[0] = lo[0] * up; f[1] = lo[1] * up; f[2] = hi[0] * up; f[3] = hi[1] * up;
}

// E2M1 codes of eight values under a block's factor, the first in the lowest four bits.  The conversion rounds to nearest even and saturates.
__device__ __forceinline__ uint32_t mx4_codes8(const float (&f)[8], int byte)
{
    const float down = byte == 255 ? 0.0f : mx_down(byte), end = byte == 253 ? 3.0f : 6.0f;      // 253: 2^126, where 4 is out of range
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_fmed3f(f[i] * down, -end, end);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.0f, 3);
    return w;
}

// ---- a lane's piece of a row: 16 bytes of bf16 (8 elements) or fp32 (4) -------------------------------------------------------
template <typename T> constexpr int kPiece = 16 / static_cast<int>(sizeof(T));

template <typename T>
__device__ __forceinline__ v4u raw_piece(const T* p) { return *reinterpret_cast<const v4u*>(p); }
template <typename T>
__device__ __forceinline__ void load_piece(const T* p, float (&f)[kPiece<T>]) { widen(raw_piece(p), f); }

__device__ __forceinline__ v4u pack_piece(const float (&f)[8])
{
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return w;
}
__device__ __forceinline__ v4u pack_piece(const float (&f)[4])
{
    v4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i]);
    return w;
}

// Gradients of a call that are more than the 256 MB memory-side cache holds go past the caches: what reads them next finds them in HBM in either case.
// (A constant of the kernel: of two stores in the branches of an `if` the compiler makes one, an ordinary one.)
constexpr int64_t kPastCaches = int64_t(256) << 20;
template <bool PAST>
__device__ __forceinline__ void store_piece(void* p, v4u w)
{
    if constexpr (PAST) __builtin_nontemporal_store(w, static_cast<v4u*>(p));
    else *static_cast<v4u*>(p) = w;
}

// codes of a piece
template <int E> struct MxCodes;
template <> struct MxCodes<8> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <> struct MxCodes<4> { typedef unsigned type; };
__device__ __forceinline__ MxCodes<8>::type mx8_piece(const float (&f)[8], float down, int byte)
{
    return MxCodes<8>::type{mx8_codes4(f[0], f[1], f[2], f[3], down, byte), mx8_codes4(f[4], f[5], f[6], f[7], down, byte)};
}
__device__ __forceinline__ MxCodes<4>::type mx8_piece(const float (&f)[4], float down, int byte) { return mx8_codes4(f[0], f[1], f[2], f[3], down, byte); }
__device__ __forceinline__ void mx8_values(MxCodes<8>::type w, float up, float (&f)[8])
{
    float lo[4], hi[4];
    mx8_values4(w[0], up, lo);
    mx8_values4(w[1], up, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = lo[i]; f[4 + i] = hi[i]; }
}
__device__ __forceinline__ void mx8_values(MxCodes<4>::type w, float up, float (&f)[4]) { mx8_values4(w, up, f); }

// ---- passes over a matrix, one piece a lane ------------------------------------------------------------------------------------
// The rows are `per_row` pieces long, a block that a row does not fill counted whole, so that a block's lanes are neighbours.
constexpr int kPieceThreads = 256;
template <typename T>
int pieces_per_row(int64_t width) { return static_cast<int>((width + MX_BLOCK - 1) / MX_BLOCK * (MX_BLOCK / kPiece<T>)); }
template <typename T>
unsigned piece_blocks(int64_t rows, int64_t width) { return static_cast<unsigned>((rows * pieces_per_row<T>(width) + kPieceThreads - 1) / kPieceThreads); }

struct Place { int64_t row; int col; bool in; };
template <int E>
__device__ __forceinline__ Place place_of(int64_t rows, int width, int per_row)
{
    const int64_t base = static_cast<int64_t>(blockIdx.x) * kPieceThreads;
    const int64_t row0 = base / per_row;                              // uniform
    const int off = static_cast<int>(base - row0 * per_row) + static_cast<int>(threadIdx.x);
    const int more = off / per_row;
    const Place p{row0 + more, (off - more * per_row) * E, false};
    return {p.row, p.col, p.row < rows && p.col < width};
}

// The sum over every 16 lanes, in all of them, in a fixed tree by DPP; and over a wave (across rows of 16 by lane swaps).
__device__ __forceinline__ float row16_sum(float v)
{
    v += dpp_move(v, std::integral_constant<int, 0xB1>{});            // quad_perm [1, 0, 3, 2]
    v += dpp_move(v, std::integral_constant<int, 0x4E>{});            // quad_perm [2, 3, 0, 1]
    v += dpp_move(v, std::integral_constant<int, 0x141>{});           // row_half_mirror
    v += dpp_move(v, std::integral_constant<int, 0x140>{});           // row_mirror
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = row16_sum(v);
    uint32_t u = __float_as_uint(v);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
    u = __float_as_uint(v);
    const auto halves = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
}

}  // namespace
}  // namespace falqon
