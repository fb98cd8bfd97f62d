// Product of microscaled 4-bit operands on the gfx950 matrix cores: c[M, N] = a[M, K] . b[N, K]^T, E2M1 codes with one power of two for
// 32 of K, fp32 accumulation.  The products of codes are exact; what is rounded is their fp32 sum and the output.
//
// Design:
//   - v_mfma_scale_f32_32x32x64_f8f6f4 with both operands E2M1: a lane holds one row's 32 codes (16 bytes) of one block, and its
//     power of two is a byte of a register, so the scales cost no arithmetic.  An instruction's two lane halves take blocks 2h + j of the four
//     that a half of a K-step has: any pairing of K is right as long as both operands use the same.
//   - A workgroup of four waves owns a tile of (64 MB) x (64 NB) outputs and walks K in steps of 256 (BK = 128 bytes of a row, whole cache lines).
//     Operand tiles go to LDS by global_load_lds in rings of S stages; the fetches of stage k + S are issued from the middle of step k on, when all
//     waves hold the rest of step k in registers (S = 2: they have until the middle of step k + 1).  They stand between the matrix instructions: a
//     wave that issues them in a row waits for the address unit and feeds no matrix core meanwhile (4096 x 4096 -> 11008: 147 us, 106 between them).
//     The exponents of two steps (16 bytes of a row) are fetched like a tile of their own.
//   - Out-of-range rows are clamped to the last one; the K tail is fetched from zeros.
//
// 4096 x 11008 -> 4096 in 84 us (4.4 PFLOP/s), 4096 x 4096 -> 11008 in 98 to 106 (3.5 to 3.8).  Of the 84 the instructions alone take 60, the fetches alone 59
// (what the L2 gives: 54 GB/s a CU), the LDS reads alone 43; all but a fifth of it overlaps.  Small products (777 x 4096 -> 4096 14 us) are bound by the L2
// and by what passes before the first and behind the last step.
#include "gemm_common.h"
#include "mx.h"

namespace falqon {
namespace {

template <int MB, int NB, int S>
constexpr int mx4_lds_bytes() { return (MB + NB) * 64 * (S * BK + S * 16); }

// the four exponent bytes that a lane needs in one step, from the eight of its row: 2h, 2h + 1, 4 + 2h, 5 + 2h
__device__ __forceinline__ int step_scales(v2i v, int half)
{
    return static_cast<int>(__builtin_amdgcn_perm(v[1], v[0], half ? 0x07060302u : 0x05040100u));
}

template <int MB, int NB, int S>
__device__ __forceinline__ void mx4_tile(const Mx4Gemm& g, int tiles_m, int tiles_n, int chunk, int bid, uint8_t* const lds)
{
    constexpr int WM = 2, WN = 2, NW = 4;
    constexpr int BM = WM * MB * 32, BN = WN * NB * 32, A_BYTES = BM * BK, B_BYTES = BN * BK;
    constexpr int PAIRS = S;                                  // buffers of exponents of two steps: S / 2 + 1 are in use at most
    uint8_t* const lds_b = lds + S * A_BYTES;
    uint8_t* const lds_sa = lds_b + S * B_BYTES;              // [PAIRS][BM][16]
    uint8_t* const lds_sb = lds_sa + PAIRS * BM * 16;             // [PAIRS][BN][16]

    // XCD x takes a run of tiles of a raster that walks panels of four tile rows, column by column
    const int xcd = bid & 7, slot = bid >> 3, tile_id = xcd * chunk + slot;
    if (slot >= chunk || tile_id >= tiles_m * tiles_n) return;
    constexpr int PH = 4;
    const int per_panel = PH * tiles_n, panel = tile_id / per_panel, rem = tile_id - panel * per_panel;
    const int ph = (tiles_m - panel * PH) < PH ? (tiles_m - panel * PH) : PH;
    const int tile_n = rem / ph, tile_m = panel * PH + (rem - tile_n * ph);

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN, half = lane >> 5;
    const int64_t m0 = static_cast<int64_t>(tile_m) * BM, n0 = static_cast<int64_t>(tile_n) * BN;
    const int64_t KB = g.K / 2, pitch = (g.K + 511) / 512 * 16;              // bytes of a row of codes, of exponents
    const int KT = static_cast<int>((KB + BK - 1) / BK);
    const int rows_a = static_cast<int>((g.M - m0) < BM ? (g.M - m0) : BM), rows_b = static_cast<int>((g.N - n0) < BN ? (g.N - n0) : BN);
    constexpr int IT_A = BM / 8 / NW, IT_B = BN / 8 / NW;                    // 1 KB fetches of a stage by one wave
    uint32_t off_a[IT_A], off_b[IT_B];
#pragma unroll
    for (int it = 0; it < IT_A; ++it) {
        const int row = (it * NW + wave) * 8 + (lane >> 3);
        off_a[it] = static_cast<uint32_t>((row < rows_a ? row : rows_a - 1) * KB) + (((lane & 7) ^ swz_kc(row)) << 4);
    }
#pragma unroll
    for (int it = 0; it < IT_B; ++it) {
        const int row = (it * NW + wave) * 8 + (lane >> 3);
        off_b[it] = static_cast<uint32_t>((row < rows_b ? row : rows_b - 1) * KB) + (((lane & 7) ^ swz_kc(row)) << 4);
    }
    const uint8_t* const base_a = g.a + m0 * KB;
    const uint8_t* const base_b = g.b + n0 * KB;
    auto dma16 = [&](const uint8_t* src, uint8_t* dst_wave_uniform) {
        __builtin_amdgcn_global_load_lds(FQ_GLOBAL_PTR(src), FQ_LDS_PTR(dst_wave_uniform), 16, 0, 0);
    };
    // The fetches of stage s by this wave: the operands' tiles, and exponents of two steps, A's of the next pair where s is odd, B's of its own
    // where it is even, so that every stage has one such fetch and none needs a branch.
    constexpr int FETCHES = IT_A + IT_B + 1;
    // (where a tile has fewer than 256 rows, several waves fetch the same ones)
    const int wave_a = wave % (BM / 64), wave_b = wave % (BN / 64), row_a = wave_a * 64 + lane, row_b = wave_b * 64 + lane;
    const uint8_t* const exp_a = g.a_exp + (m0 + (row_a < rows_a ? row_a : rows_a - 1)) * pitch;
    const uint8_t* const exp_b = g.b_exp + (n0 + (row_b < rows_b ? row_b : rows_b - 1)) * pitch;
    const int last_pair = static_cast<int>(pitch / 16) - 1;
    struct Stage { const uint8_t *pa, *pb; int s; };
    auto stage_of = [&](int s) {
        const int64_t k0 = static_cast<int64_t>(s) * BK;
        return Stage{opaque_uniform(base_a + k0), opaque_uniform(base_b + k0), s};
    };
    auto fetch_one = [&](const Stage& f, int j, bool whole) {
        auto inside = [&](int it) { return static_cast<int64_t>(f.s) * BK + (((lane & 7) ^ swz_kc((it * NW + wave) * 8 + (lane >> 3))) << 4) < KB; };
        const int slot = f.s & (S - 1);
        if (j < IT_A) {
            dma16(whole || inside(j) ? f.pa + off_a[j] : g_zero16, lds + slot * A_BYTES + (j * NW + wave) * 1024);
        } else if (j < IT_A + IT_B) {
            const int it = j - IT_A;
            dma16(whole || inside(it) ? f.pb + off_b[it] : g_zero16, lds_b + slot * B_BYTES + (it * NW + wave) * 1024);
        } else {
            const int next = (f.s + 1) >> 1, pair = next < last_pair ? next : last_pair;      // also that of an even s
            const bool of_a = f.s & 1;
            dma16((of_a ? exp_a : exp_b) + pair * 16, of_a ? lds_sa + ((next & (PAIRS - 1)) * BM + wave_a * 64) * 16 : lds_sb + ((next & (PAIRS - 1)) * BN + wave_b * 64) * 16);
        }
    };
    auto fetch = [&](int s, int from) {
        const Stage f = stage_of(s);
#pragma unroll
        for (int j = 0; j < FETCHES; ++j)
            if (j >= from) fetch_one(f, j, false);
    };
    // Of the fetches of stage k + S the first are issued in the second half of step k, which frees the slot, and the others, where the ring
    // leaves the time, in the first half of step k + 1.
    constexpr int EARLY = S > 2 ? FETCHES / 2 : FETCHES;
    const int steady_steps = static_cast<int>(KB / BK) - S;   // steps kt whose stage kt + S lies fully inside K

    // LDS reads are done, and fetches but those of the last n stages
    auto wait_stages = [&](int n) {
        static_assert((S - 1) * FETCHES < 64, "fetches are counted in six bits");
        auto but = [](int left) { return (left & 15) | ((left >> 4) << 14) | 0x70; };        // vmcnt left, lgkmcnt 0
        if (S > 6 && n >= 6) __builtin_amdgcn_s_waitcnt(but(S > 6 ? 6 * FETCHES : 0));
        else if (S > 4 && n >= 4) __builtin_amdgcn_s_waitcnt(but(S > 4 ? 4 * FETCHES : 0));
        else if (S > 3 && n >= 3) __builtin_amdgcn_s_waitcnt(but(S > 3 ? 3 * FETCHES : 0));
        else if (S > 2 && n >= 2) __builtin_amdgcn_s_waitcnt(but(2 * FETCHES));
        else if (n >= 1) __builtin_amdgcn_s_waitcnt(but(FETCHES));
        else __builtin_amdgcn_s_waitcnt(but(0));
    };

    v16f acc[MB][NB];
#pragma unroll
    for (int mi = 0; mi < MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NB; ++ni)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0.0f;

    v4i af[2][MB][2], bf[2][NB][2];                           // [half of a step][block of 32 rows][instruction]
    int sa[MB], sb[NB];                                       // exponents of a step
    auto read_frag = [&](const uint8_t* tile, int row, int kh, v4i (&f)[2]) {
        const int cb = kh * 4 + half * 2, sw = swz_kc(row);
        f[0] = *reinterpret_cast<const v4i*>(tile + row * BK + ((cb ^ sw) << 4));
        f[1] = *reinterpret_cast<const v4i*>(tile + row * BK + (((cb + 1) ^ sw) << 4));
    };
    auto read_half = [&](int s, int kh, int which) {
        if (which < NB) read_frag(lds_b + (s & (S - 1)) * B_BYTES, wn * NB * 32 + which * 32 + (lane & 31), kh, bf[kh][which]);
        else if (which < NB + MB) read_frag(lds + (s & (S - 1)) * A_BYTES, wm * MB * 32 + (which - NB) * 32 + (lane & 31), kh, af[kh][which - NB]);
    };
    // (All LDS reads of the loop are of types that the compiler takes to differ from what the fetches write: of a struct like uint2 it does not know,
    // and waits for every fetch in flight before such a read.)
    auto read_exps = [&](int s, v2i (&ra)[MB], v2i (&rb)[NB]) {
        const int at = (s >> 1) & (PAIRS - 1), byte = (s & 1) * 8;
#pragma unroll
        for (int i = 0; i < MB; ++i) ra[i] = *reinterpret_cast<const v2i*>(lds_sa + at * (BM * 16) + (wm * MB * 32 + i * 32 + (lane & 31)) * 16 + byte);
#pragma unroll
        for (int i = 0; i < NB; ++i) rb[i] = *reinterpret_cast<const v2i*>(lds_sb + at * (BN * 16) + (wn * NB * 32 + i * 32 + (lane & 31)) * 16 + byte);
    };
    auto take_exps = [&](const v2i (&ra)[MB], const v2i (&rb)[NB]) {
#pragma unroll
        for (int i = 0; i < MB; ++i) sa[i] = step_scales(ra[i], half);
#pragma unroll
        for (int i = 0; i < NB; ++i) sb[i] = step_scales(rb[i], half);
    };
    auto wide = [](v4i v) { return v8i{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; };
    constexpr int N_MFMA = 2 * MB * NB, N_FRAG = MB + NB;     // of a half step
    // the weight operand first: a lane's accumulators are then four consecutive columns of one row
    auto mfma = [&](auto kh_tag, auto j_tag, int mi, int ni, const int (&ra)[MB], const int (&rb)[NB]) {
        constexpr int KH = decltype(kh_tag)::value, J = decltype(j_tag)::value;
        acc[mi][ni] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(bf[KH][ni][J]), wide(af[KH][mi][J]), acc[mi][ni], 4, 4, KH * 2 + J, rb[ni], KH * 2 + J, ra[mi]);
    };

    dma16(exp_a, lds_sa + wave_a * 1024);
#pragma unroll
    for (int s = 0; s < S - 1; ++s)
        if (s < KT) fetch(s, 0);
    if (steady_steps > 0) {
        const Stage f = stage_of(S - 1);
#pragma unroll
        for (int j = 0; j < EARLY; ++j) fetch_one(f, j, true);
    } else if (S - 1 < KT) {
        fetch(S - 1, 0);
    }
    constexpr int BEHIND = EARLY < FETCHES ? S - 2 : S - 1;   // whole stages that are in flight behind the first
    wait_stages(KT - 1 < BEHIND ? KT - 1 : BEHIND);           // the first has landed
    barrier_lds_only();
#pragma unroll
    for (int f = 0; f < N_FRAG; ++f) read_half(0, 0, f);
    v2i next_a[MB], next_b[NB];
    read_exps(0, next_a, next_b);
    take_exps(next_a, next_b);

    constexpr int PER = (2 * N_FRAG + N_MFMA - 1) / N_MFMA;                  // operands read beside an instruction
    // The instructions of a half step, with the reads of half `kh` of stage s and the fetches of a stage beside them.
    auto half_step = [&](auto kh_tag, int s, int kh, auto from_tag, auto to_tag, const Stage& f) {
        constexpr int FROM = decltype(from_tag)::value, COUNT = decltype(to_tag)::value - FROM;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int mi = 0; mi < MB; ++mi)
#pragma unroll
                for (int ni = 0; ni < NB; ++ni) {
                    if (j == 0) mfma(kh_tag, std::integral_constant<int, 0>{}, mi, ni, sa, sb);
                    else mfma(kh_tag, std::integral_constant<int, 1>{}, mi, ni, sa, sb);
                    const int q = (j * MB + mi) * NB + ni;
#pragma unroll
                    for (int u = q * COUNT / N_MFMA; u < (q + 1) * COUNT / N_MFMA; ++u) fetch_one(f, FROM + u, true);
#pragma unroll
                    for (int u = 0; u < PER; ++u) read_half(s, kh, q * PER + u);
                    __builtin_amdgcn_sched_barrier(0);
                }
    };
    auto k_step = [&](int kt, auto steady) {
        constexpr bool STEADY = decltype(steady)::value;
        using None = std::integral_constant<int, 0>;
        using Early = std::integral_constant<int, STEADY ? EARLY : 0>;
        using All = std::integral_constant<int, STEADY ? FETCHES : 0>;
        half_step(std::integral_constant<int, 0>{}, kt, 1, Early{}, All{}, stage_of(kt + S - 1));
        // the rest of step kt is in registers, stage kt + 1 in LDS, for every wave
        const int behind = KT - 2 - kt;
        wait_stages(STEADY || behind > S - 2 ? S - 2 : behind > 0 ? behind : 0);
        barrier_lds_only();
        if (!STEADY && kt + S < KT) fetch(kt + S, 0);
        // (behind the last step these read what is left in the next slot, and nothing uses it)
        read_exps(kt + 1, next_a, next_b);                    // used behind the instructions that follow
        half_step(std::integral_constant<int, 1>{}, kt + 1, 0, None{}, Early{}, stage_of(kt + S));
        take_exps(next_a, next_b);
    };
    int kt = 0;
    for (; kt < steady_steps; ++kt) k_step(kt, std::true_type{});
    if (EARLY < FETCHES && kt > 0) fetch(kt + S - 1, EARLY);
    for (; kt < KT; ++kt) k_step(kt, std::false_type{});

    // ---- epilogue: every wave converts its part, through LDS of its own, and stores whole pieces of rows -------------------
    __syncthreads();                                          // all operand reads are done
    auto epilogue = [&](auto is_f32) {
        constexpr bool F32 = decltype(is_f32)::value;
        constexpr int ES = F32 ? 4 : 2, PITCH = NB * 32 * ES + 16, SEGS = NB * 32 * ES / 16, COLS = 16 / ES;
        constexpr int BLOCKS = F32 && MB == 4 ? 2 : MB;       // blocks of 32 rows at a time
        static_assert(NW * BLOCKS * 32 * PITCH <= mx4_lds_bytes<MB, NB, S>(), "the waves' parts fit");
        uint8_t* const out = static_cast<uint8_t*>(g.c);
        uint8_t* const part = lds + wave * (BLOCKS * 32 * PITCH);
#pragma unroll
        for (int m = 0; m < MB; m += BLOCKS) {
#pragma unroll
            for (int mi = m; mi < m + BLOCKS; ++mi) {
                uint8_t* const srow = part + ((mi - m) * 32 + (lane & 31)) * PITCH;
#pragma unroll
                for (int ni = 0; ni < NB; ++ni) {
                    v16f t = acc[mi][ni];
                    asm volatile("" : "+v"(t));               // one block at a time leaves the accumulation registers
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = ni * 32 + q * 8 + half * 4;
                        if (F32) *reinterpret_cast<float4*>(srow + c * 4) = make_float4(t[4 * q], t[4 * q + 1], t[4 * q + 2], t[4 * q + 3]);
                        else *reinterpret_cast<uint2*>(srow + c * 2) = make_uint2(pack_bf16x2(t[4 * q], t[4 * q + 1]), pack_bf16x2(t[4 * q + 2], t[4 * q + 3]));
                    }
                }
            }
#pragma unroll
            for (int it = 0; it < BLOCKS * 32 * SEGS / 64; ++it) {
                const int i = it * 64 + lane, srw = i / SEGS, seg = i % SEGS;
                const int64_t row = m0 + wm * (MB * 32) + m * 32 + srw, col = n0 + wn * (NB * 32) + seg * COLS;
                if (row < g.M && col < g.N) {
                    // Past the caches at any size: the next reader loses nothing by it.  us of gate and up on one input and the SwiGLU product of them, with
                    // these stores and with ordinary ones: 64 tokens 4096 -> 11008 22.6, 22.6; 777 70.4, 71.6; 4096 275.5, 274.1; 8192 x 5120 -> 13824 757, 780.
                    typedef unsigned v4u __attribute__((ext_vector_type(4)));
                    __builtin_nontemporal_store(*reinterpret_cast<const v4u*>(part + srw * PITCH + seg * 16), reinterpret_cast<v4u*>(out + (row * g.N + col) * ES));
                }
            }
        }
    };
    if (g.c_is_f32) epilogue(std::true_type{});
    else epilogue(std::false_type{});
}

template <int MB, int NB, int S>
__global__ void __launch_bounds__(256)
mx4_gemm_kernel(const Mx4Gemm g, int tiles_m, int tiles_n, int chunk)
{
    __shared__ __attribute__((aligned(1024))) uint8_t lds[mx4_lds_bytes<MB, NB, S>()];
    mx4_tile<MB, NB, S>(g, tiles_m, tiles_n, chunk, blockIdx.x, lds);
}

template <int MB, int NB, int S>
void launch(const Mx4Gemm& g, hipStream_t stream)
{
    const int tiles_m = static_cast<int>((g.M + 64 * MB - 1) / (64 * MB)), tiles_n = static_cast<int>((g.N + 64 * NB - 1) / (64 * NB));
    const int chunk = (tiles_m * tiles_n + 7) / 8;
    mx4_gemm_kernel<MB, NB, S><<<static_cast<unsigned>(chunk * 8), 256, 0, stream>>>(g, tiles_m, tiles_n, chunk);
}

}  // namespace

// The smallest tiles of which there is one for a CU at most (a tile's steps take the longer the larger it is, but 64 x 64 only a quarter of 256 x 256
// for a sixteenth of the work); beyond, two 128 x 128 a CU with rings of two, and the largest.  us by tile 64x64, 128x64, 128x128, the same two a CU,
// 256x256: 128 x 4096 -> 4096 7.7, 10.2, 12.9, 15.0, 28.4; 512 x 4096 -> 4096 13.1, 11.6, 13.5, 16.0, 31.3; 777 x 4096 -> 4096 22.2, 20.3, 15.3, 17.1, 32.4;
// 2048 x 4096 -> 4096 42.3, 38.3, 27.3, 24.1, 33.5; 3000 x 4096 -> 4096 62.1, 56.5, 39.4, 38.6, 36.6; 1009 x 3744 -> 560 8.2, 11.5, 15.7, 17.6, 33.1.
hipError_t launch_mx4_gemm(const Mx4Gemm& g, hipStream_t stream)
{
    auto tiles = [&](int64_t rows, int64_t columns) { return ((g.M + rows - 1) / rows) * ((g.N + columns - 1) / columns); };
    if (tiles(64, 64) <= 256) launch<1, 1, 4>(g, stream);
    else if (tiles(128, 64) <= 256) launch<2, 1, 4>(g, stream);
    else if (tiles(128, 128) <= 256) launch<2, 2, 4>(g, stream);
    else if (tiles(128, 128) <= 512) launch<2, 2, 2>(g, stream);
    else launch<4, 4, 2>(g, stream);
    return hipGetLastError();
}

}  // namespace falqon
