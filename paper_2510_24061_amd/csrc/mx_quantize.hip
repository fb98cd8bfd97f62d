// Microscaled codes of a matrix, 8 bits (E4M3) or 4 (E2M1), and the values they stand for (definitions in mx_common.h).
//
// One pass, bound by bytes (bf16: 2 + 33/32 or 2 + 17/32 bytes an element): a lane takes 16 bytes, the lanes of a block of 32 columns
// are neighbours.  No maximum over the tensor is needed, so there is no second pass as in the per-tensor quantizer.  4096 x 4096 from bf16 to
// 4 bits 9.5 us (4.5 TB/s), to 8 bits 10.4; 8192 x 13824 54 and 64 (5.3 and 5.4 TB/s).  Values of 8-bit codes 9.6 and 61 us; of 4-bit ones, whose bytes are read one by
// one, 12.4 and 72 (floors 8.3 and 56): they are for tests and for looking at codes, no layer reads them.
#include "mx_common.h"
#include "mx.h"

namespace falqon {
namespace {

// bytes of a row of exponents: of 4-bit codes filled up to 16, for the product's fetches
template <bool FOUR>
__device__ __forceinline__ int exp_pitch(int width) { return FOUR ? (width + 511) / 512 * 16 : (width + MX_BLOCK - 1) / MX_BLOCK; }

__device__ __forceinline__ uint32_t mx4_piece(const float (&f)[8], int byte) { return mx4_codes8(f, byte); }
__device__ __forceinline__ uint16_t mx4_piece(const float (&f)[4], int byte)
{
    const float both[8] = {f[0], f[1], f[2], f[3], 0.0f, 0.0f, 0.0f, 0.0f};
    return static_cast<uint16_t>(mx4_codes8(both, byte));
}

template <typename T, bool FOUR>
__global__ void __launch_bounds__(kPieceThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t ld_x, int64_t rows, int width, int per_row, uint8_t* __restrict__ q, uint8_t* __restrict__ exps)
{
    constexpr int E = kPiece<T>;
    const Place at = place_of<E>(rows, width, per_row);
    v4u raw = {};
    if (at.in) raw = raw_piece(x + at.row * ld_x + at.col);
    const int byte = mx_exponent<FOUR ? MX_E2M1_EMAX : MX_E4M3_EMAX>(block_max_bits<E>(abs_max_bits(raw, x)));
    if (!at.in) return;
    float f[E];
    widen(raw, f);
    if constexpr (FOUR) {
        *reinterpret_cast<decltype(mx4_piece(f, byte))*>(q + (at.row * width + at.col) / 2) = mx4_piece(f, byte);
    } else {
        *reinterpret_cast<typename MxCodes<E>::type*>(q + at.row * width + at.col) = mx8_piece(f, mx_down(byte), byte);
    }
    if (at.col % MX_BLOCK == 0) {
        uint8_t* const to = exps + at.row * exp_pitch<FOUR>(width) + at.col / MX_BLOCK;
        *to = static_cast<uint8_t>(byte);
        if (FOUR && at.col + MX_BLOCK == width)                       // the rest of the row's exponents
            for (int i = 1; i < exp_pitch<FOUR>(width) - at.col / MX_BLOCK; ++i) to[i] = 0;
    }
}

template <typename T, bool FOUR>
__global__ void __launch_bounds__(kPieceThreads)
mx_values_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ exps, int64_t rows, int width, int per_row, T* __restrict__ x, int64_t ld_x)
{
    constexpr int E = kPiece<T>;
    const Place at = place_of<E>(rows, width, per_row);
    if (!at.in) return;
    float f[E];
    const float up = mx_up(exps[at.row * exp_pitch<FOUR>(width) + at.col / MX_BLOCK]);
    if constexpr (FOUR) {
        const uint8_t* const p = q + (at.row * width + at.col) / 2;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const uint32_t code = (p[i / 2] >> (4 * (i & 1))) & 15u, a = code & 7u;
            // 0, 0.5, 1, 1.5, 2, 3, 4, 6: one bit of significand, one subnormal
            const float v = a < 2 ? 0.5f * static_cast<float>(a) : __uint_as_float(((a >> 1) + 126u) << 23 | (a & 1u) << 22);
            f[i] = (code & 8u ? -v : v) * up;
        }
    } else {
        mx8_values(*reinterpret_cast<const typename MxCodes<E>::type*>(q + at.row * width + at.col), up, f);
    }
    *reinterpret_cast<v4u*>(x + at.row * ld_x + at.col) = pack_piece(f);
}

template <typename T, bool FOUR>
void quantize(const void* x, int64_t rows, int64_t cols, int64_t ld_x, uint8_t* q, uint8_t* exps, hipStream_t stream)
{
    mx_quantize_kernel<T, FOUR><<<piece_blocks<T>(rows, cols), kPieceThreads, 0, stream>>>(static_cast<const T*>(x), ld_x, rows, static_cast<int>(cols), pieces_per_row<T>(cols), q, exps);
}
template <typename T, bool FOUR>
void values(const uint8_t* q, const uint8_t* exps, int64_t rows, int64_t cols, void* x, int64_t ld_x, hipStream_t stream)
{
    mx_values_kernel<T, FOUR><<<piece_blocks<T>(rows, cols), kPieceThreads, 0, stream>>>(q, exps, rows, static_cast<int>(cols), pieces_per_row<T>(cols), static_cast<T*>(x), ld_x);
}

}  // namespace

hipError_t launch_mx_quantize(const void* x, bool f32, int64_t rows, int64_t cols, int64_t ld_x, bool four, uint8_t* q, uint8_t* exps, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    if (f32) four ? quantize<float, true>(x, rows, cols, ld_x, q, exps, stream) : quantize<float, false>(x, rows, cols, ld_x, q, exps, stream);
    else four ? quantize<uint16_t, true>(x, rows, cols, ld_x, q, exps, stream) : quantize<uint16_t, false>(x, rows, cols, ld_x, q, exps, stream);
    return hipGetLastError();
}

hipError_t launch_mx_values(const uint8_t* q, const uint8_t* exps, int64_t rows, int64_t cols, bool four, void* x, bool f32, int64_t ld_x, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    if (f32) four ? values<float, true>(q, exps, rows, cols, x, ld_x, stream) : values<float, false>(q, exps, rows, cols, x, ld_x, stream);
    else four ? values<uint16_t, true>(q, exps, rows, cols, x, ld_x, stream) : values<uint16_t, false>(q, exps, rows, cols, x, ld_x, stream);
    return hipGetLastError();
}

}  // namespace falqon
