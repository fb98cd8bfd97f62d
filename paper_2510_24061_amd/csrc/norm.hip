// RMS norms on both sides of a block, with the block's channel gate and residual scale, forward and backward.
//
//   u = b, or b rstd_b w_post with rstd_b = 1 / sqrt(mean(b^2) + eps)
//   s = round(x + (scale gate) u),  h = round(s rstd w) with rstd = 1 / sqrt(mean(s^2) + eps), of the rounded s
//
//   ds = ds_in + rstd (w dh - s^ mean(w dh s^)),  s^ = s rstd                 (dx)
//   du = scale gate ds;  db = du, or rstd_b (w_post du - b^ mean(w_post du b^)),  b^ = b rstd_b
//   dw = sum_t dh s^,  dw_post = sum_t du b^,  dgate = scale sum_t ds u
//
// Everything is bound by the bytes that it has to move, so each tensor goes through a lane's registers once: a row belongs to one
// wave or to some of a workgroup, 16 bytes a lane and piece, and its sums run over lanes by DPP and over waves through LDS.  Sums,
// statistics and weight gradients are fp32.  The backward pass keeps a workgroup on several rows, so that the sums over tokens stay in registers;
// one partial for each workgroup is left, and a second launch adds them in order (no atomics: the result does not change from run to run).
// 8192 x 5120 in bf16 with both norms, gate and checkpoints: forward 89 us (4.75 TB/s), backward 84 us (5.05 TB/s, 79 + 5); a copy reaches 5.15.
// Forward in fp32 (floor): 4096 x 5120 with everything 93 us (74), with a plain branch 68 (66); 8192 x 4096 118 (118) and 99 (105).
// Rows of more than 8192 columns (fp32: 4096) take two or four pieces a lane in the backward pass and keep the sums over tokens in LDS.
// With both norms, gate and checkpoints: fp32 4096 x 5120 81 us (floor 73; 111 with the sums in registers, which spill), bf16
// 4096 x 16384 162 (130; 522).  bf16 4096 x 10240 with a plain branch 83 from checkpoints (74), 85 without (82).
#include "mx_common.h"
#include "norm.h"

namespace falqon {
namespace {

constexpr int kMaxWaves = 16;

// Sums over the waves of a row.  Consecutive calls take turns between two slots, so one barrier each is enough.
struct RowSum {
    float (*slots)[kMaxWaves];
    int turn = 0;
    __device__ __forceinline__ float operator()(float v, int wave, int first, int waves)
    {
        v = wave_sum(v);
        if (waves == 1) return v;
        float* const s = slots[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[wave] = v;
        barrier_lds_written();
        // every row of 16 lanes reads the waves' sums at once and adds them by DPP (one after the other, each waits 0.1 us for LDS)
        const int lane = threadIdx.x & 15;
        return row16_sum(lane < waves ? s[first + lane] : 0.0f);
    }
};

__device__ __forceinline__ float element(const float* p) { return *p; }
__device__ __forceinline__ float element(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }

__device__ __forceinline__ float inverse_root(float sum_sq, float width, float eps) { return 1.0f / sqrtf(sum_sq / width + eps); }

// checkpoint of a piece.  The codes are next read in the backward pass: they go past the caches (101 us to 98 at 8192 x 5120).
template <typename T>
__device__ __forceinline__ void store_codes(v4u raw, uint8_t* q, uint8_t* exps, int64_t row, int d, int col, bool in)
{
    constexpr int E = kPiece<T>;
    const int byte = mx_exponent<MX_E4M3_EMAX>(block_max_bits<E>(abs_max_bits(raw, static_cast<const T*>(nullptr))));   // zeros outside
    if (!in) return;
    float f[E];
    widen(raw, f);
    __builtin_nontemporal_store(mx8_piece(f, mx_down(byte), byte), reinterpret_cast<typename MxCodes<E>::type*>(q + row * d + col));
    if (col % MX_BLOCK == 0) exps[row * ((d + MX_BLOCK - 1) / MX_BLOCK) + col / MX_BLOCK] = static_cast<uint8_t>(byte);
}

template <typename T, int P, bool POST>
__global__ void __launch_bounds__(1024)
norm_fwd_kernel(const NormFwd a, int waves, int rows_per_group)
{
    constexpr int E = kPiece<T>;
    __shared__ float slots[2][kMaxWaves];
    RowSum row_sum{slots};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = wave / waves, first = group * waves;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * rows_per_group + group;
    const bool live = row < a.T;
    const int d = static_cast<int>(a.d);
    const float width = static_cast<float>(d);
    const T *const x = static_cast<const T*>(a.x) + row * a.ld_x, *const b = static_cast<const T*>(a.b) + row * a.ld_b;
    int col[P];
    bool in[P];
    v4u raw_x[P] = {}, raw_b[P] = {}, raw_post[P] = {}, raw_gate[P] = {}, raw_w[P] = {};
#pragma unroll
    for (int p = 0; p < P; ++p) {                                     // all of them at once: later ones would wait behind the stores
        col[p] = ((p * waves + wave - first) * 64 + lane) * E;
        in[p] = live && col[p] < d;
        if (!in[p]) continue;
        raw_x[p] = raw_piece(x + col[p]);
        if (a.b) raw_b[p] = raw_piece(b + col[p]);
        if (POST) raw_post[p] = raw_piece(static_cast<const T*>(a.w_post) + col[p]);
        if (a.gate) raw_gate[p] = raw_piece(static_cast<const T*>(a.gate) + col[p]);
        raw_w[p] = raw_piece(static_cast<const T*>(a.w) + col[p]);
    }
    float xs[P][E], u[P][E];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        widen(raw_x[p], xs[p]);
        widen(raw_b[p], u[p]);
    }
    if (a.b) {
        if (a.bq)
#pragma unroll
            for (int p = 0; p < P; ++p) store_codes<T>(raw_b[p], a.bq, a.b_exp, row, d, col[p], in[p]);
        if (POST) {
            float sq = 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < E; ++i) sq += u[p][i] * u[p][i];
            const float rb = inverse_root(row_sum(sq, wave, first, waves), width, a.eps);
            if (live && wave == first && lane == 0) a.rstd_b[row] = rb;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float w[E];
                widen(raw_post[p], w);
#pragma unroll
                for (int i = 0; i < E; ++i) u[p][i] = u[p][i] * rb * w[i];
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float c[E];
#pragma unroll
            for (int i = 0; i < E; ++i) c[i] = 1.0f;
            if (a.gate) widen(raw_gate[p], c);
#pragma unroll
            for (int i = 0; i < E; ++i) xs[p][i] = __fadd_rn(xs[p][i], __fmul_rn(u[p][i], a.scale * c[i]));
            raw_x[p] = pack_piece(xs[p]);                             // s as it is held, in the place of x
            widen(raw_x[p], xs[p]);
            if (in[p]) *reinterpret_cast<v4u*>(static_cast<T*>(a.s) + row * d + col[p]) = raw_x[p];
        }
    }
    if (a.sq)
#pragma unroll
        for (int p = 0; p < P; ++p) store_codes<T>(raw_x[p], a.sq, a.s_exp, row, d, col[p], in[p]);
    float sq = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < E; ++i) sq += xs[p][i] * xs[p][i];
    const float r = inverse_root(row_sum(sq, wave, first, waves), width, a.eps);
    if (live && wave == first && lane == 0) a.rstd[row] = r;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!in[p]) continue;
        float w[E], h[E];
        widen(raw_w[p], w);
#pragma unroll
        for (int i = 0; i < E; ++i) h[i] = xs[p][i] * r * w[i];
        *reinterpret_cast<v4u*>(static_cast<T*>(a.h) + row * d + col[p]) = pack_piece(h);
    }
}

// The address of a piece: what all lanes share, and a lane's column as an offset of 32 bits, which takes one register for all tensors
// and not two for each.
template <typename V, typename T>
__device__ __forceinline__ V* piece_at(T* row, uint32_t col)
{
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte_t;
    return reinterpret_cast<V*>(reinterpret_cast<byte_t*>(row) + col * static_cast<uint32_t>(sizeof(T)));
}

// A piece of a saved tensor, as it is or as its checkpoint, on the way and then as values.
template <typename T, bool CODES> struct Saved {
    static constexpr int E = kPiece<T>;
    v4u raw;
    __device__ __forceinline__ void load(const void* v, const uint8_t*, int64_t row, int, int64_t ld, uint32_t col) { raw = *piece_at<const v4u>(static_cast<const T*>(v) + row * ld, col); }
    __device__ __forceinline__ void values(float (&f)[E]) const { widen(raw, f); }
};
template <typename T> struct Saved<T, true> {
    static constexpr int E = kPiece<T>;
    typename MxCodes<E>::type raw;
    uint8_t byte;
    __device__ __forceinline__ void load(const void* v, const uint8_t* exps, int64_t row, int d, int64_t, uint32_t col)
    {
        raw = *piece_at<const typename MxCodes<E>::type>(static_cast<const uint8_t*>(v) + row * d, col);
        byte = *piece_at<const uint8_t>(exps + row * ((d + MX_BLOCK - 1) / MX_BLOCK), col / MX_BLOCK);
    }
    __device__ __forceinline__ void values(float (&f)[E]) const { mx8_values(raw, mx_up(byte), f); }
};

// MODE: what there is of a branch.  0 none; 1 b plain (db = scale ds); 2 a gate (b is read); 3 a norm of b, and a gate or none
// A row's pieces are asked for while the row before is worked on (AHEAD).
template <typename T, int P, bool CODES, int MODE>
__global__ void __launch_bounds__(1024)
norm_bwd_kernel(const NormBwd a, int waves, int rows_per_group, float* __restrict__ partial)
{
    constexpr int E = kPiece<T>;
    // One piece a lane: sums and weights stay in registers, and the next row's pieces are on the way.  Two: the sums stand in LDS; in bf16, whose pieces
    // have twice the columns, rows with b are not asked for ahead and their weights come from the caches again for each (otherwise they spill, 4096 x 10240
    // with both norms 248 us against 112).  What spills all the same: two pieces of bf16 from checkpoints with a plain branch, asked for ahead (5 registers),
    // and four (fp32 above 8192 columns) with a branch, not asked for ahead (4 to 121; 4096 x 16384 370 us, and 490 with the weights from the caches).
    constexpr bool HELD = P == 1, AHEAD = P * E < 16 || (P == 2 && MODE < 2), KEPT = AHEAD || P == 4;
    __shared__ float slots[2][kMaxWaves];
    extern __shared__ __attribute__((aligned(16))) float gathered[];  // [d] where a workgroup has several rows
    RowSum row_sum{slots};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, group = wave / waves, first = group * waves;
    const uint32_t d = static_cast<uint32_t>(a.d);
    const float width = static_cast<float>(d);
    uint32_t col[P];
    float dw[P][E] = {}, q[P][E] = {};                                // sums over rows of dh s^, of ds b or ds b^
    __shared__ v4f sums[HELD ? 1 : MODE >= 2 ? 2 : 1][HELD ? 1 : P * E / 4][HELD ? 1 : 1024];      // the same, each lane's own
    auto add = [&](int vector, int p, float (&v)[P][E], const float (&f)[E]) {
        if constexpr (HELD) {
#pragma unroll
            for (int i = 0; i < E; ++i) v[p][i] += f[i];
        } else {
#pragma unroll
            for (int i = 0; i < E; i += 4) sums[vector][(p * E + i) / 4][threadIdx.x] += v4f{f[i], f[i + 1], f[i + 2], f[i + 3]};
        }
    };
    if constexpr (!HELD)
#pragma unroll
        for (int k = 0; k < (MODE >= 2 ? 2 : 1) * P * E / 4; ++k) sums[k / (P * E / 4)][k % (P * E / 4)][threadIdx.x] = v4f{};
#pragma unroll
    for (int p = 0; p < P; ++p) col[p] = static_cast<uint32_t>((p * waves + wave - first) * 64 + lane) * E;
    struct Pieces {
        v4u dh[P], ds[P];
        Saved<T, CODES> s[P], b[MODE >= 2 ? P : 1];
        float rstd, rstd_b;
    };
    auto load_row = [&](int64_t row) {
        Pieces v{};
        if (row >= a.T) return v;
        v.rstd = a.rstd[row];
        if (MODE == 3) v.rstd_b = a.rstd_b[row];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (col[p] >= d) continue;
            v.s[p].load(a.s, a.s_exp, row, d, a.ld_s, col[p]);
            v.dh[p] = *piece_at<const v4u>(static_cast<const T*>(a.dh) + row * a.ld_dh, col[p]);
            if (a.ds) v.ds[p] = *piece_at<const v4u>(static_cast<const T*>(a.ds) + row * a.ld_ds, col[p]);
            if constexpr (MODE >= 2) v.b[p].load(a.b, a.b_exp, row, d, a.ld_b, col[p]);
        }
        return v;
    };
    // The weights' pieces stay in registers: loads come back in order, so one inside the loop would be waited for behind the next row's and the
    // stores of the last.
    v4u raw_w[P], raw_gate[P], raw_post[P];
    auto load_w = [&] {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            raw_w[p] = v4u{};
            if (col[p] < d) raw_w[p] = *piece_at<const v4u>(static_cast<const T*>(a.w), col[p]);
        }
    };
    auto load_branch_weights = [&] {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            raw_gate[p] = raw_post[p] = v4u{};
            if (col[p] >= d) continue;
            if (a.gate) raw_gate[p] = *piece_at<const v4u>(static_cast<const T*>(a.gate), col[p]);
            if (MODE == 3) raw_post[p] = *piece_at<const v4u>(static_cast<const T*>(a.w_post), col[p]);
        }
    };
    if (KEPT) {
        load_w();
        load_branch_weights();
    }
    const int64_t stride = static_cast<int64_t>(gridDim.x) * rows_per_group;
    int64_t base = static_cast<int64_t>(blockIdx.x) * rows_per_group;
    Pieces next{};
    if (AHEAD) next = load_row(base + group);
    for (; base < a.T; base += stride) {
        const int64_t row = base + group;
        const bool live = row < a.T;
        const Pieces now = AHEAD ? next : load_row(row);
        if (AHEAD) next = load_row(row + stride);
        if (!KEPT) load_w();
        const float r = now.rstd;
        float hat[P][E], g[P][E];                                     // s^; w dh
        float dot = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float dh[E], w[E], part[E];
            now.s[p].values(hat[p]);
            widen(now.dh[p], dh);
            widen(raw_w[p], w);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                hat[p][i] *= r;
                g[p][i] = w[i] * dh[i];
                part[i] = dh[i] * hat[p][i];
                dot += g[p][i] * hat[p][i];
            }
            add(0, p, dw, part);
        }
        if (!KEPT) load_branch_weights();
        dot = row_sum(dot, wave, first, waves) / width;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float in[E];
            widen(now.ds[p], in);                                     // zeros where there is none
#pragma unroll
            for (int i = 0; i < E; ++i) g[p][i] = in[i] + r * (g[p][i] - hat[p][i] * dot);     // ds
            if (live && col[p] < d) *piece_at<v4u>(static_cast<T*>(a.dx) + row * d, col[p]) = pack_piece(g[p]);
        }
        if (MODE == 0) continue;
        const float rb = now.rstd_b;
        float dot_b = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float c[E], wp[E], part[E];
#pragma unroll
            for (int i = 0; i < E; ++i) c[i] = 1.0f;
            if (a.gate) widen(raw_gate[p], c);
            if constexpr (MODE >= 2) now.b[p].values(hat[p]);
            if (MODE == 3) widen(raw_post[p], wp);
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float ds = g[p][i], du = ds * (a.scale * c[i]);
                g[p][i] = du;
                if (MODE == 3) {
                    hat[p][i] *= rb;                                  // b^
                    g[p][i] = wp[i] * du;
                    dot_b += g[p][i] * hat[p][i];
                }
                part[i] = ds * hat[p][i];
            }
            if (MODE >= 2) add(1, p, q, part);
        }
        if (MODE == 3) dot_b = row_sum(dot_b, wave, first, waves) / width;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (!(live && col[p] < d)) continue;
            if (MODE == 3)
#pragma unroll
                for (int i = 0; i < E; ++i) g[p][i] = rb * (g[p][i] - hat[p][i] * dot_b);
            if (a.db) *piece_at<v4u>(static_cast<T*>(a.db) + row * d, col[p]) = pack_piece(g[p]);
        }
    }
    // the workgroup's partials of dw and of q, [vector][workgroup][d]
    auto leave = [&](const float (&v)[P][E], int vector) {
        float* const out = partial + (static_cast<int64_t>(vector) * gridDim.x + blockIdx.x) * d;
        for (int k = 0; k < rows_per_group; ++k) {                    // the rows' sums one after the other
            if (group == k) {
                float* const to = k + 1 < rows_per_group ? gathered : out;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (col[p] >= d) continue;
#pragma unroll
                    for (int i = 0; i < E; i += 4) {
                        float4 f = make_float4(v[p][i], v[p][i + 1], v[p][i + 2], v[p][i + 3]);
                        if constexpr (!HELD) {
                            const v4f sum = sums[vector][(p * E + i) / 4][threadIdx.x];
                            f = make_float4(sum[0], sum[1], sum[2], sum[3]);
                        }
                        if (k > 0) {
                            const float4 g4 = *reinterpret_cast<const float4*>(gathered + col[p] + i);
                            f = make_float4(f.x + g4.x, f.y + g4.y, f.z + g4.z, f.w + g4.w);
                        }
                        *reinterpret_cast<float4*>(to + col[p] + i) = f;
                    }
                }
            }
            if (rows_per_group > 1) __syncthreads();
        }
    };
    if (a.dw) leave(dw, 0);
    if (MODE >= 2 && (a.dgate || a.dw_post)) leave(q, 1);
}

// The partials' sums in the order of the workgroups, within sixteen interleaved shares: dw, or q with what it stands for,
//   dgate = scale sum_t ds u = scale w_post q (scale q without a norm of b),  dw_post = sum_t scale gate ds b^ = scale gate q
constexpr int kShares = 16;
template <typename T>
__global__ void __launch_bounds__(64 * kShares)
norm_sum_kernel(const float* __restrict__ partial, int parts, const NormBwd a)
{
    __shared__ float shares[kShares][64];
    const int d = static_cast<int>(a.d);
    if (blockIdx.y == 0 ? !a.dw : !(a.dgate || a.dw_post)) return;
    const int column = blockIdx.x * 64 + (threadIdx.x & 63), share = threadIdx.x >> 6;
    float sum = 0.0f;
    if (column < d) {
        const float* const v = partial + static_cast<int64_t>(blockIdx.y) * parts * d + column;
#pragma unroll 8
        for (int k = share; k < parts; k += kShares) sum += v[static_cast<int64_t>(k) * d];
    }
    shares[share][threadIdx.x & 63] = sum;
    __syncthreads();
    if (share != 0 || column >= d) return;
#pragma unroll
    for (int k = 1; k < kShares; ++k) sum += shares[k][threadIdx.x];
    if (blockIdx.y == 0) {
        a.dw[column] = sum;
        return;
    }
    sum *= a.scale;
    if (a.dgate) a.dgate[column] = a.w_post ? sum * element(static_cast<const T*>(a.w_post) + column) : sum;
    if (a.dw_post) a.dw_post[column] = a.gate ? sum * element(static_cast<const T*>(a.gate) + column) : sum;
}

struct FwdShape { int P, waves, rows; };                              // pieces a lane, waves a row, rows a workgroup
template <typename T>
FwdShape fwd_shape(int64_t d)
{
    constexpr int E = kPiece<T>;
    const int pieces = static_cast<int>(d) / E;
    int P = 1, waves = (pieces + 63) / 64;
    while (waves > 4 && P < 16 / E) { P *= 2; waves = (pieces + 64 * P - 1) / (64 * P); }
    return {P, waves, waves >= 4 ? 1 : 4 / waves};
}

template <typename T, bool POST>
void run_fwd(const NormFwd& a, hipStream_t stream)
{
    constexpr int E = kPiece<T>;
    const auto [P, waves, rows] = fwd_shape<T>(a.d);
    const unsigned grid = static_cast<unsigned>((a.T + rows - 1) / rows);
    const int threads = 64 * waves * rows;
    if (P == 1) norm_fwd_kernel<T, 1, POST><<<grid, threads, 0, stream>>>(a, waves, rows);
    else if (P == 2) norm_fwd_kernel<T, 2, POST><<<grid, threads, 0, stream>>>(a, waves, rows);
    else if constexpr (E == 4) norm_fwd_kernel<T, 4, POST><<<grid, threads, 0, stream>>>(a, waves, rows);
}

template <typename T, int P, bool CODES, int MODE>
void run_bwd(const NormBwd& a, float* partial, hipStream_t stream)
{
    constexpr int E = kPiece<T>;
    const int pieces = static_cast<int>(a.d) / E, waves = (pieces + 64 * P - 1) / (64 * P);
    int rows = waves < 8 ? 8 / waves : 1;
    const int64_t enough = (a.T + kNormGroups - 1) / kNormGroups;
    if (rows > enough) rows = static_cast<int>(enough);
    int64_t groups = (a.T + rows - 1) / rows;
    // one workgroup a CU where it has more than eight waves, as no second one finds registers beside it (8192 x 5120: 92 us with 512, 85 with 256)
    const int64_t most = waves * rows > 8 ? kNormGroups / 2 : kNormGroups;
    if (groups > most) groups = most;
    const size_t lds = rows > 1 ? static_cast<size_t>(a.d) * sizeof(float) : 0;      // up to 8 KB: a row is then four waves at the most
    norm_bwd_kernel<T, P, CODES, MODE><<<static_cast<unsigned>(groups), 64 * waves * rows, lds, stream>>>(a, waves, rows, partial);
    if (a.dw || a.dgate || a.dw_post)
        norm_sum_kernel<T><<<dim3(static_cast<unsigned>((a.d + 63) / 64), 2), 64 * kShares, 0, stream>>>(partial, static_cast<int>(groups), a);
}

template <typename T, bool CODES, int MODE>
void bwd_by_pieces(const NormBwd& a, float* partial, hipStream_t stream)
{
    constexpr int E = kPiece<T>;
    const int64_t pieces = a.d / E;
    if (pieces <= 64 * kMaxWaves) run_bwd<T, 1, CODES, MODE>(a, partial, stream);
    else if (E == 8 || pieces <= 64 * 2 * kMaxWaves) run_bwd<T, 2, CODES, MODE>(a, partial, stream);
    else if constexpr (E == 4) run_bwd<T, 4, CODES, MODE>(a, partial, stream);
}

template <typename T, bool CODES>
void bwd_by_mode(const NormBwd& a, float* partial, hipStream_t stream)
{
    if (a.w_post) bwd_by_pieces<T, CODES, 3>(a, partial, stream);
    else if (a.dgate) bwd_by_pieces<T, CODES, 2>(a, partial, stream);
    else if (a.db) bwd_by_pieces<T, CODES, 1>(a, partial, stream);
    else bwd_by_pieces<T, CODES, 0>(a, partial, stream);
}

}  // namespace

int64_t norm_fwd_threads(int64_t T, int64_t d, bool f32)
{
    const FwdShape s = f32 ? fwd_shape<float>(d) : fwd_shape<uint16_t>(d);
    return (T + s.rows - 1) / s.rows * (64 * s.waves * s.rows);
}

hipError_t launch_norm_fwd(const NormFwd& a, bool f32, hipStream_t stream)
{
    if (f32) a.w_post ? run_fwd<float, true>(a, stream) : run_fwd<float, false>(a, stream);
    else a.w_post ? run_fwd<uint16_t, true>(a, stream) : run_fwd<uint16_t, false>(a, stream);
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormBwd& a, bool f32, float* partial, hipStream_t stream)
{
    const bool codes = a.s_exp != nullptr;
    if (f32) codes ? bwd_by_mode<float, true>(a, partial, stream) : bwd_by_mode<float, false>(a, partial, stream);
    else codes ? bwd_by_mode<uint16_t, true>(a, partial, stream) : bwd_by_mode<uint16_t, false>(a, partial, stream);
    return hipGetLastError();
}

}  // namespace falqon
