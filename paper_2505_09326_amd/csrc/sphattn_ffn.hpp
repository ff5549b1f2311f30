// The gated feed-forward product of a layer and its gradients, for gfx950.
//
//   A = X Wg^T      U = X Wu^T      H = act(A) U
//   dA = dH U act'(A)      dB = dH act(A)      dX = dA Wg + dB Wu      dWg = dA^T X      dWu = dB^T X
//
// Both projections run in one tile (Form::Two of the tile products): a lane holds the same element of A and of U, so the product of the two needs no
// memory.  The gradients form A and U once more, into dA and dB, so that nothing has to be kept between the two calls (8 T F bytes as fp32; what 16 bits of
// them leave of dA and dB would be most of the error).  Past D of about 950 that takes longer than writing and reading them would: 4 T F D operations of 8192 x 2048 x 8192 some
// 450 us at the products' rate, 16 T F bytes some 210 at memory's; below it less.  dX is one sum over 2 F (Form::Sum), dWg and dWu are two over T.
//
// dA and dB are rounded once to the storage type, which is what the matrix instructions take; sums are in fp32 throughout.  That rounding is as large as the results'
// own, of 1.7e-3 in bf16 it makes 2.3e-3 against 64 bits on average over the terms; where there are few of them, up to 2^18 values, chance made 2.5e-3 and more of it,
// and they are kept in two 16-bit parts: twice the products, beside which launches and the weights' bytes are most of the time there (gradients of 256 x 1024 x 1024 in bf16 42.7 us,
// in one part 34.8; 64 x 2048 x 4096 56 and 49).  fp16: they are scaled by powers of two that keep them in the type's range whatever the gradients' size, by each row for dX and by each
// column for dW, as two pairs.
// fp32: A and U as three products of two fp16 parts with a power of two per row, the gradients as six of three bf16 parts, as the vocabulary loss has them.
// Bound by the matrix pipes: 8192 rows, D = 2048, F = 8192 in bf16 forward 487 us (1129 TFLOP/s; a library product of 8192^3 1227), dA and dB 545, dX 436 (1261), dWg and dWu
// 422 (1303).  What the gate's tiles lose to that is their end, exponentials and stores beside which no other tile's products run (8 rounds).
#pragma once
#include "sphattn_tiles.hpp"

namespace sphattn {

enum class Gate { Silu, Gelu, Relu };

// act(a) and its slope.  The exponential's argument is rounded to fp32: |a| 2^-24 of the exponential, which EXACT (fp32 storage) makes up for.
// Exponentials are of numbers that are not positive and end in 0, below 2^-126: what a far gate is multiplied with vanishes, however large the gate (a mask of the type's
// lowest value has act and slope 0), and an infinite one is NaN where the formula's 0 times infinity is.
template <Gate G, bool EXACT>
__device__ __forceinline__ void gate(float a, float& act, float& slope)
{
    auto exp_of = [](float x) {                    // e^x, x <= 0
        x = fmaxf(x, -200.f);                      // (the correction has no infinite argument)
        const float y = x * kLog2e;
        float e = __builtin_amdgcn_exp2f(y);
        if constexpr (EXACT) e = __builtin_fmaf(e, kLn2 * (__builtin_fmaf(x, kLog2e, -y) + x * 1.925963033e-8f), e);   // (log2(e) and what fp32 leaves of it)
        return e;
    };
    if constexpr (G == Gate::Relu) {
        act = a <= 0.f ? 0.f : a;
        slope = a > 0.f ? 1.f : 0.f;
    } else if constexpr (G == Gate::Silu) {
        if constexpr (EXACT) {
            // 1 / (1 + e^-a) and what is left of 1
            const float e = exp_of(-__builtin_fabsf(a)), large = 1.f / (1.f + e), small = e * large;
            const float s = a < 0.f ? small : large, rest = a < 0.f ? large : small;
            act = a * s;
            slope = s * __builtin_fmaf(a, rest, 1.f);
        } else {                                   // (an infinite exponential gives zeros; 1 - s is off by 2^-24 where s is near 1)
            const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -kLog2e));
            act = a * s;
            slope = __builtin_fmaf(act, 1.f - s, s);
        }
    } else {
        const float half = exp_of(-0.5f * a * a);
        float below;                               // the normal distribution's share below a
        if constexpr (EXACT) below = 0.5f * erfcf(a * -0.70710678118654752f);
        else {
            // e^(x^2) erfc(x) as t times a polynomial in t = 1 / (1 + 0.475 x), fitted to x = 0 .. 9.4, where the exponential ends: 1.1e-5 of itself at most and 2.5e-8 of
            // the share (what fp32 makes of it 1.5e-7), so that the tail keeps either 16-bit type's bits all the way (a formula of 1.5e-7 whatever the size, as Abramowitz and Stegun
            // 7.1.26, is off by 5e-4 of the tail at -4, 2e-2 at -10)
            const float x = __builtin_fabsf(a) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.475f, x, 1.f));
            float p = 0.0850622207f;
            p = __builtin_fmaf(p, t, -0.395078987f);
            p = __builtin_fmaf(p, t, 0.542703986f);
            p = __builtin_fmaf(p, t, -0.0715403333f);
            p = __builtin_fmaf(p, t, 0.314265907f);
            p = __builtin_fmaf(p, t, 0.255825222f);
            p = __builtin_fmaf(p, t, 0.268761963f);
            const float tail = 0.5f * p * t * half;
            below = a < 0.f ? tail : 1.f - tail;
        }
        act = a * below;
        slope = __builtin_fmaf(a * 0.39894228040143268f, half, below);
        if (a != a) act = slope = a;
    }
}

struct FfnArgs {
    Operand G, U, X;                               // Wg, Wu, X as the products take them
    const int *g_exp, *u_exp, *x_exp;              // fp32: the powers of two that each row was divided by (or kEndless) ...
    const float *g_whole, *u_whole, *x_whole; int D;   // ... and the rows as they are
    int k, tiles_p, T, F;
    void* H;                                       // forward: [T,F]
    const void* dH;                                // backward: [T,F]
    unsigned short *dA, *dB; long long part; int ld;   // [T,ld], in parts (fp32 three, few values two)
    // fp16: factors of dA and dB by row, and the second pair with powers of two by column, dA's in the lower half of an int
    const float* row_up; const int* col_up; unsigned short *dA_all, *dB_all;
    const float *x_norm, *g_norm;                  // relu's slopes: the norms of X's and Wg's rows
};

// Eight (fp32: four) neighbouring elements of a row of F: what of it is in the row
template <Store S>
__device__ __forceinline__ void store_piece(void* out, size_t at, i32x4 w, int left, bool wide)
{
    if (left <= 0) return;
    if (wide) store16<S, true>(out, at, w, per16<S>());
    else store16<S, false>(out, at, w, left);
}

// the corner of A and U of this wave from rows of fp32 as they are, for the rare tile that meets a row with an infinite element (see whole_logits)
template <class T>
__device__ __forceinline__ void whole_projections(f32x4 (&acc)[T::FP][T::FQ], const FfnArgs& a, int fw, int qw)
{
    const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
    const float *pat[T::FP], *qat[T::FQ];          // (rows behind the last one take the last one's place: their results are not looked at)
#pragma unroll
    for (int i = 0; i < T::FP; ++i) pat[i] = (i & 1 ? a.u_whole : a.g_whole) + (size_t)min(fw + i / 2 * 16 + n16, a.F - 1) * a.D;
#pragma unroll
    for (int j = 0; j < T::FQ; ++j) {
        qat[j] = a.x_whole + (size_t)min(qw + 16 * j + n16, a.T - 1) * a.D;
#pragma unroll
        for (int i = 0; i < T::FP; ++i) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll 1
    for (int k = g; k < a.D + g; k += 4) {
        float w[T::FP], x[T::FQ];
#pragma unroll
        for (int i = 0; i < T::FP; ++i) w[i] = k < a.D ? pat[i][k] : 0.f;
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) x[j] = k < a.D ? qat[j][k] : 0.f;
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int j = 0; j < T::FQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[j], acc[i][j], 0, 0, 0);
    }
}

// relu's slope beside 0: which side A is on is for the sum in 64 bits to say, not for what fp32 has lost of it (of 249 x 6144 values one was on the other side: 1.2e-3
// of dX, 1.7e-3 of dWg).  What a sum may be off by goes by its terms, |x| |w| at most, however small it is itself: a matrix instruction was never more than 4.8 2^-24 of its terms'
// and its addend's size off (10^6 sums of six kinds), and the partial sums of one that ends near 0 are half of the terms' size at most, so that n of them make (2.5 n + 5) 2^-24.
// Values below that, an exact 0 among them, are formed again: few of a fragment four at a time, each by sixteen lanes, more of them with all of the fragment by the fp64 matrix
// instruction, so that no data (sparse rows, weights that take an offset of X away) costs more than that.  (D = 2048: 4.3e-4 of all values where both are normally distributed.)
constexpr float kSlopeSteps = 3.f, kSlopeRest = 8.f, kSlopeParts = 13.f;   // 2^-24 of |x| |w| each: per instruction, at least, for what parts of fp32 leave out
// Of a fragment's 256 values: gradients of 2048 x 1024 x 2048 in bf16 with 16, 32 and 256 of them 201, 283 and 1607 us four at a time, 295, 281 and 280 with the instruction (without any
// 108); in fp32 441, 559 and 2376, 604, 605 and 594 (326)
constexpr int kSlopeMany = 32;
typedef __attribute__((ext_vector_type(4))) double f64x4;

template <class T, Store S>
__device__ __forceinline__ void settle_signs(f32x4 (&acc)[T::FP][T::FQ], const FfnArgs& a, int fw, int qw, bool whole)
{
    constexpr int R = T::FP / 2 * 4;               // values of a row in a lane
    static_assert(R * T::FQ <= 64, "");
    constexpr bool F32 = S == Store::F32;
    constexpr int N = per16<S>();
    const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
    // (fp32 as it is: four k an instruction)
    const float steps = F32 && whole ? (float)((a.D + 3) / 4) : (float)((a.k + kStepK - 1) / kStepK);
    const float off = 0x1p-24f * (kSlopeSteps * steps + kSlopeRest + (F32 ? kSlopeParts : 0.f));
    uint64_t open = 0;                             // by value: not settled
    float x_norm[T::FQ];
#pragma unroll
    for (int j = 0; j < T::FQ; ++j) x_norm[j] = qw + 16 * j + n16 < a.T ? a.x_norm[qw + 16 * j + n16] : 0.f;
#pragma unroll
    for (int i = 0; i < R / 4; ++i) {
        const int f = fw + 16 * i + 4 * g;
        const f32x4 g_norm = *(const f32x4*)(a.g_norm + f);   // (the array goes on to a tile's end)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float norm = f + r < a.F ? g_norm[r] : 0.f;
#pragma unroll
            for (int j = 0; j < T::FQ; ++j) {
                // (and what is lost below the normal numbers; a row of zeros has sums of 0)
                const float size = __builtin_fabsf(acc[2 * i][j][r]), top = __builtin_fmaf(x_norm[j] * norm, off, 0x1p-132f);
                const bool near = size <= top && size < __builtin_inff() && fminf(x_norm[j], norm) > 0.f;
                open |= (uint64_t)near << (j * R + 4 * i + r);
            }
        }
    }
    if (!__ballot(open != 0)) return;
    asm("" : "+v"(open));                          // (seen through, each of its bits is kept as a comparison's own result, in scratch)
    const uint64_t found = open;
    uint64_t above = 0;                            // by value: greater than 0
    // 16 bytes of row q of X or row f of Wg, zeros behind its end
    const int end = F32 ? a.D : a.k;
    auto piece = [&](bool of_x, int row, int k, float (&x)[N]) {
        i32x4 w = {0, 0, 0, 0};
        if (k < end) {
            if constexpr (F32) w = load16<S, false>(of_x ? a.x_whole : a.g_whole, (size_t)row * end + k, end - k, (size_t)((of_x ? a.T : a.F) - row) * end - k);
            else w = *(const i32x4*)((of_x ? a.X : a.G).data + (size_t)row * (of_x ? a.X : a.G).ld + (size_t)k * 2);
        }
        widen16<S>(w, x);
    };
#pragma unroll 1
    for (int n = 0; n < R / 4 * T::FQ; ++n) {      // fragments with many
        const uint32_t mine = (uint32_t)(open >> (n * 4)) & 15;
        int count = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) count += __builtin_popcountll(__ballot(mine >> r & 1));
        if (count <= kSlopeMany) continue;
        // (the instruction leaves row 4 r + g of its first operand in register r of lane group g: there goes column 4 g + r)
        const int f = min(fw + n % (R / 4) * 16 + 4 * (n16 & 3) + (n16 >> 2), a.F - 1), q = min(qw + n / (R / 4) * 16 + n16, a.T - 1);
        f64x4 sum = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
        for (int k = g * N; k < end + g * N; k += 4 * N) {
            float w[N], x[N];
            piece(false, f, k, w);
            piece(true, q, k, x);
#pragma unroll
            for (int i = 0; i < N; ++i) sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)w[i], (double)x[i], sum, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) above |= (uint64_t)(sum[r] > 0.0) << (n * 4 + r);
        open &= ~((uint64_t)15 << (n * 4));
    }
    for (uint64_t lanes; (lanes = __ballot(open != 0)) != 0;) {
        const int first = open ? __builtin_ctzll(open) : 0;
        int who[4], which[4], my_who = -1, my_which = 0;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            who[m] = lanes ? __builtin_ctzll(lanes) : -1;
            lanes &= lanes - 1;
            which[m] = __builtin_amdgcn_readlane(first, max(who[m], 0));
            my_who = g == m ? who[m] : my_who;
            my_which = g == m ? which[m] : my_which;
        }
        const int j = my_which / R, v = my_which % R, at = max(my_who, 0);
        const int f = min(fw + v / 4 * 16 + 4 * (at >> 4) + (v & 3), a.F - 1), q = min(qw + 16 * j + (at & 15), a.T - 1);
        double sum = 0.0;
#pragma unroll 2
        for (int k = n16 * N; k < end; k += 16 * N) {
            float w[N], x[N];
            piece(false, f, k, w);
            piece(true, q, k, x);
#pragma unroll
            for (int i = 0; i < N; ++i) sum = __builtin_fma((double)w[i], (double)x[i], sum);
        }
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
        const uint64_t positive = __ballot(sum > 0.0);
#pragma unroll
        for (int m = 0; m < 4; ++m)
            if (lane == who[m]) {
                open &= open - 1;
                above |= (positive >> (16 * m) & 1) << which[m];
            }
    }
#pragma unroll
    for (int j = 0; j < T::FQ; ++j)
#pragma unroll
        for (int v = 0; v < R; ++v) {
            const float x = acc[v / 4 * 2][j][v & 3], size = __builtin_fabsf(x);
            acc[v / 4 * 2][j][v & 3] = !(found >> (j * R + v) & 1) ? x : above >> (j * R + v) & 1 ? fmaxf(size, 0x1p-126f) : -size;
        }
}

// A tile of BP / 2 columns of F and BQ rows: H, or dA and dB.  TWO: these in two 16-bit parts
template <class T, Store S, bool BACK, bool TWO = false>
__global__ __launch_bounds__(T::THREADS, T::FP * T::FQ > 32 ? 1 : 2)
void ffn_gate_kernel(FfnArgs a, int act)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    SPH_LDS unsigned char* const smem = (SPH_LDS unsigned char*)smem_raw;
    constexpr bool F32 = S == Store::F32, HALF = S == Store::F16;
    const int tiles_q = (a.T + T::BQ - 1) / T::BQ;
    const TileAt tile = tile_of(xcd_contiguous_id(blockIdx.x, a.tiles_p * tiles_q), a.tiles_p, tiles_q);
    const int f0 = __builtin_amdgcn_readfirstlane(tile.p) * (T::BP / 2), q0 = __builtin_amdgcn_readfirstlane(tile.q) * T::BQ;
    Product<T, HALF || F32, false, false, F32 ? 3 : 1, Form::Two> prod;
    prod.run(a.G, a.X, f0, q0, 0, a.k, smem, a.U);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int fw = f0 + wave % T::WAVES_P * (T::FP / 2) * 16, qw = q0 + wave / T::WAVES_P * T::FQ * 16;   // this wave's corner
    bool whole = false;
    if constexpr (F32) {
        int qe[T::FQ];
        bool endless = false;
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) endless |= (qe[j] = a.x_exp[min(qw + 16 * j + n16, a.T - 1)]) == kEndless;
#pragma unroll
        for (int i = 0; i < T::FP; ++i) {          // (the arrays go on to a tile's end; what stands there changes nothing: the products are 0)
            const int f = fw + i / 2 * 16 + 4 * g;
            const i32x4 pe = *(const i32x4*)((i & 1 ? a.u_exp : a.g_exp) + f);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                endless |= pe[r] == kEndless && f + r < a.F;
#pragma unroll
                for (int j = 0; j < T::FQ; ++j) prod.acc[i][j][r] = __builtin_ldexpf(prod.acc[i][j][r], pe[r] + qe[j]);
            }
        }
        whole = __ballot(endless) != 0;
        if (whole) whole_projections<T>(prod.acc, a, fw, qw);
    }
    if constexpr (BACK)
        if (act == (int)Gate::Relu) settle_signs<T, S>(prod.acc, a, fw, qw, whole);
    static_assert(T::FP % 4 == 0, "");
    constexpr int E = store_bytes<S>();
    const void* const rows = BACK ? a.dH : a.H;
    const bool wide = (((uintptr_t)rows | (uintptr_t)((size_t)a.F * E)) & 15) == 0;
    // 16-bit: two fragments at a time, whose lanes exchange halves, so that each has eight neighbouring columns of one and 16 bytes to load or store.
    // dH of the whole corner is asked for at once: a row block at a time, each behind the last one's arithmetic, took dA and dB of 8192 x 2048 x 8192 from 545 us to 560.
    constexpr int PIECES = F32 ? T::FP / 2 : T::FP / 4;
    i32x4 dh[T::FQ][PIECES];
    if constexpr (BACK) {
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) {
            const size_t row = (size_t)min(qw + 16 * j + n16, a.T - 1) * a.F;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int at = F32 ? fw + 16 * i + 4 * g : fw + 16 * (2 * i + (g & 1)) + 8 * (g >> 1);
                dh[j][i] = i32x4{0, 0, 0, 0};
                if (at < a.F)
                    dh[j][i] = wide ? load16<S, true>(a.dH, row + at, per16<S>(), per16<S>()) : load16<S, false>(a.dH, row + at, a.F - at, (size_t)a.T * a.F - row - at);
            }
        }
    }
    i32x4 col_up[T::FP / 2];                       // (the array goes on to a tile's end: what stands there changes nothing, the values are 0)
    if constexpr (BACK && HALF) {
        if (a.dA_all) {
#pragma unroll
            for (int i = 0; i < T::FP / 2; ++i) col_up[i] = *(const i32x4*)(a.col_up + fw + 16 * i + 4 * g);
        }
    }
    auto corner = [&](auto gate_of) {
        constexpr Gate G = decltype(gate_of)::value;
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) {
            const int q = qw + 16 * j + n16;
            const size_t row = (size_t)min(q, a.T - 1) * a.F;
            float up = 1.f;
            if constexpr (BACK && HALF) up = a.row_up[min(q, a.T - 1)];
#pragma unroll
            for (int i = 0; i < T::FP / 2; i += 2) {
                // where this lane's piece of the two fragments stands (fp32: a piece of each)
                const int f = F32 ? fw + 16 * i + 4 * g : fw + 16 * (i + (g & 1)) + 8 * (g >> 1);
                float d[2][4];
                if constexpr (BACK) {
                    if constexpr (F32) {
                        widen16<S>(dh[j][i], d[0]);
                        widen16<S>(dh[j][i + 1], d[1]);
                    } else {
                        const i32x4 w = dh[j][i / 2], h = join_fragments(i32x2{w[0], w[1]}, i32x2{w[2], w[3]});   // (the exchange is its own inverse)
                        float x[8];
                        widen16<S>(h, x);
#pragma unroll
                        for (int r = 0; r < 4; ++r) d[0][r] = x[r], d[1][r] = x[4 + r];
                    }
                }
                float y[2][4], z[2][4];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float u = prod.acc[2 * (i + s) + 1][j][r];
                        float value, slope;
                        gate<G, F32>(prod.acc[2 * (i + s)][j][r], value, slope);
                        if constexpr (BACK) {
                            y[s][r] = d[s][r] * (u * slope);       // (dH U may be past fp32's range beside a closed gate)
                            z[s][r] = d[s][r] * value;
                        } else {
                            y[s][r] = value * u;
                        }
                    }
                auto pack = [&](const float (&v)[2][4], float by) {
                    return join_fragments(i32x2{pack2<HALF>(v[0][0] * by, v[0][1] * by), pack2<HALF>(v[0][2] * by, v[0][3] * by)},
                                          i32x2{pack2<HALF>(v[1][0] * by, v[1][1] * by), pack2<HALF>(v[1][2] * by, v[1][3] * by)});
                };
                if constexpr (!BACK) {
                    if constexpr (F32) {
#pragma unroll
                        for (int s = 0; s < 2; ++s)
                            if (q < a.T) store_piece<S>(a.H, row + f + 16 * s, narrow16<S>(y[s]), a.F - f - 16 * s, wide);
                    } else {
                        const i32x4 w = pack(y, 1.f);
                        if (q < a.T) store_piece<S>(a.H, row + f, w, a.F - f, wide);
                    }
                } else {
                    const size_t at = (size_t)q * a.ld + (F32 ? fw + 16 * (i + (g & 1)) + 8 * (g >> 1) : f);
                    const bool in = q < a.T && (F32 ? fw + 16 * (i + (g & 1)) + 8 * (g >> 1) : f) < a.ld;
                    if constexpr (F32) {
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            i32x2 part[2][3];      // [fragment][part]
#pragma unroll
                            for (int s = 0; s < 2; ++s) split3(m ? z[s] : y[s], part[s]);
#pragma unroll
                            for (int p = 0; p < 3; ++p) {
                                const i32x4 w = join_fragments(part[0][p], part[1][p]);
                                if (in) *(i32x4*)((m ? a.dB : a.dA) + p * a.part + at) = w;
                            }
                        }
                    } else {
                        auto put = [&](unsigned short* to, const float (&v)[2][4], float by) {
                            const i32x4 w = pack(v, by);
                            if (in) *(i32x4*)(to + at) = w;
                            if constexpr (TWO) {
                                auto rest = [&](const float (&x)[4]) {
                                    return i32x2{pack2_rest<HALF>(x[0] * by, x[1] * by, pack2<HALF>(x[0] * by, x[1] * by)),
                                                 pack2_rest<HALF>(x[2] * by, x[3] * by, pack2<HALF>(x[2] * by, x[3] * by))};
                                };
                                const i32x4 r = join_fragments(rest(v[0]), rest(v[1]));
                                if (in) *(i32x4*)(to + a.part + at) = r;
                            }
                        };
                        put(a.dA, y, up);
                        put(a.dB, z, up);
                        if constexpr (HALF) {
                            if (a.dA_all) {
#pragma unroll
                                for (int s = 0; s < 2; ++s)
#pragma unroll
                                    for (int r = 0; r < 4; ++r) {
                                        const int e = col_up[i + s][r];
                                        y[s][r] = __builtin_ldexpf(y[s][r], e << 16 >> 16);
                                        z[s][r] = __builtin_ldexpf(z[s][r], e >> 16);
                                    }
                                put(a.dA_all, y, 1.f);
                                put(a.dB_all, z, 1.f);
                            }
                        }
                    }
                }
            }
        }
    };
    if (act == (int)Gate::Silu) corner(std::integral_constant<Gate, Gate::Silu>{});
    else if (act == (int)Gate::Gelu) corner(std::integral_constant<Gate, Gate::Gelu>{});
    else corner(std::integral_constant<Gate, Gate::Relu>{});
}

// ---- few rows -----------------------------------------------------------------------------------------------

// H for few rows, at most 64, where reading the weights is most of the time: they go from memory straight into registers, once.  A workgroup takes sixteen
// columns of F, its waves a share of D each, in runs of 256 bytes of a row; lane (i, g) holds 16 bytes of row i of each operand (any order of k
// will do if both have it).  fp32 on the fp32 matrix instruction, as it is.  (One row of 1024 x 4096 in bf16 5.1 us, both weights at 3.3 TB/s.)
template <int FQ> constexpr int ffn_row_waves() { return FQ == 4 ? 4 : 8; }

template <Store S, int FQ, bool WIDE>
__global__ __launch_bounds__(64 * ffn_row_waves<FQ>())
void ffn_rows_kernel(const void* __restrict__ X, const void* __restrict__ Wg, const void* __restrict__ Wu, void* __restrict__ H, int T, int D, int F, int act)
{
    constexpr int WAVES = ffn_row_waves<FQ>(), N = per16<S>(), STEP = 4 * N, RUN = 4;   // STEP: k of one 16-byte load of all lanes; RUN of them neighbours
    __shared__ f32x4 sums[WAVES][2][FQ][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int f0 = (int)blockIdx.x * 16;
    const size_t pat = (size_t)min(f0 + n16, F - 1) * D, all = (size_t)F * D, all_x = (size_t)T * D;
    size_t qat[FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) qat[j] = (size_t)min(16 * j + n16, T - 1) * D;
    f32x4 acc[2][FQ];
#pragma unroll
    for (int j = 0; j < FQ; ++j) acc[0][j] = acc[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto load = [&](const void* from, size_t at, int k, size_t end) {
        if (k >= D) return i32x4{0, 0, 0, 0};
        return load16<S, WIDE>(from, at + k, D - k, end - at - k);
    };
    i32x4 next[2][RUN];
    auto fetch = [&](int k) {
#pragma unroll
        for (int c = 0; c < RUN; ++c) {
            next[0][c] = load(Wg, pat, k + c * STEP + g * N, all);
            next[1][c] = load(Wu, pat, k + c * STEP + g * N, all);
        }
    };
    const int first = wave * RUN * STEP;
    fetch(first);
    for (int k = first; k < D; k += WAVES * RUN * STEP) {
        i32x4 w[2][RUN], x[RUN][FQ];
#pragma unroll
        for (int c = 0; c < RUN; ++c) {
            w[0][c] = next[0][c], w[1][c] = next[1][c];
#pragma unroll
            for (int j = 0; j < FQ; ++j) x[c][j] = load(X, qat[j], k + c * STEP + g * N, all_x);
        }
        fetch(k + WAVES * RUN * STEP);
#pragma unroll
        for (int c = 0; c < RUN; ++c)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < FQ; ++j) {
                    if constexpr (S == Store::F32) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[m][j] = mfma_f32(w[m][c], x[c][j], r, acc[m][j]);
                    } else {
                        acc[m][j] = mfma16x16<S == Store::F16>(w[m][c], x[c][j], acc[m][j]);
                    }
                }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < FQ; ++j) sums[wave][m][j][lane] = acc[m][j];
    __syncthreads();
    // lane (t, g) of wave j: columns 4 g .. + 3 of row 16 j + t
    if (wave >= FQ) return;
    f32x4 A = sums[0][0][wave][lane], U = sums[0][1][wave][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) A += sums[w][0][wave][lane], U += sums[w][1][wave][lane];
    const int t = 16 * wave + n16;
    if (t >= T) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int f = f0 + 4 * g + r;
        if (f >= F) return;
        float value, slope;
        if (act == (int)Gate::Silu) gate<Gate::Silu, S == Store::F32>(A[r], value, slope);
        else if (act == (int)Gate::Gelu) gate<Gate::Gelu, S == Store::F32>(A[r], value, slope);
        else gate<Gate::Relu, S == Store::F32>(A[r], value, slope);
        store_el<S>(H, (size_t)t * F + f, value * U[r]);
    }
}

// ---- sums of the gradients ------------------------------------------------------------------------------------

struct FfnSum {
    Operand P, P2, Q, Q2;
    int k, tiles_p, slices;
    void* out; int out_ld, out_cols, out_rows;     // in the storage type, where there is one slice
    float* part; int part_ld;                      // else [slices][out_rows][part_ld]
    const float* row_down;                         // fp16
};

// dX [T,D] = dA Wg + dB Wu
template <class T, Store S, bool DX, bool TWO>
__device__ __forceinline__ void ffn_sum_tile(const FfnSum& a, int id, SPH_LDS unsigned char* smem)
{
    constexpr bool F32 = S == Store::F32;
    const int tiles_q = (a.out_rows + T::BQ - 1) / T::BQ;
    const TileAt tile = tile_of(xcd_contiguous_id(id, a.tiles_p * tiles_q * a.slices), a.tiles_p, tiles_q);
    const int p0 = __builtin_amdgcn_readfirstlane(tile.p) * T::BP, q0 = __builtin_amdgcn_readfirstlane(tile.q) * T::BQ;
    const int per_slice = __builtin_amdgcn_readfirstlane(((a.k + kStepK - 1) / kStepK + a.slices - 1) / a.slices) * kStepK;
    const int slice = __builtin_amdgcn_readfirstlane(tile.slice);
    const int k0 = min(a.k, slice * per_slice), k1 = min(a.k, k0 + per_slice);
    Product<T, S == Store::F16, true, !DX, F32 ? 6 : TWO ? 2 : 1, DX ? Form::Sum : Form::One> prod;
    prod.run(a.P, a.Q, p0, q0, k0, k1, smem, a.P2, a.Q2);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int pw = p0 + wave % T::WAVES_P * T::FP * 16, qw = q0 + wave / T::WAVES_P * T::FQ * 16;
    const bool wide = (((uintptr_t)a.out | (uintptr_t)((size_t)a.out_ld * store_bytes<S>())) & 15) == 0;
#pragma unroll
    for (int j = 0; j < T::FQ; ++j) {
        const int q = qw + 16 * j + n16;
        const bool in = q < a.out_rows;
        if (a.slices > 1) {
#pragma unroll
            for (int i = 0; i < T::FP; ++i) {
                const int p = pw + 16 * i + 4 * g;
                if (in && p < a.part_ld) *(f32x4*)(a.part + ((size_t)slice * a.out_rows + q) * a.part_ld + p) = prod.acc[i][j];
            }
            continue;
        }
        float by = 1.f;
        if constexpr (S == Store::F16) by = a.row_down ? a.row_down[min(q, a.out_rows - 1)] : 1.f;
        const size_t row = (size_t)q * a.out_ld;
#pragma unroll
        for (int i = 0; i < T::FP; i += 2) {
            const f32x4 x = prod.acc[i][j] * by, z = prod.acc[i + 1][j] * by;
            if constexpr (F32) {
                const int p = pw + 16 * i + 4 * g;
                if (in) store_piece<S>(a.out, row + p, __builtin_bit_cast(i32x4, x), a.out_cols - p, wide);
                if (in) store_piece<S>(a.out, row + p + 16, __builtin_bit_cast(i32x4, z), a.out_cols - p - 16, wide);
            } else {
                const i32x4 o = join_fragments(i32x2{pack2<S == Store::F16>(x[0], x[1]), pack2<S == Store::F16>(x[2], x[3])},
                                               i32x2{pack2<S == Store::F16>(z[0], z[1]), pack2<S == Store::F16>(z[2], z[3])});
                const int p = pw + 16 * (i + (g & 1)) + 8 * (g >> 1);
                if (in) store_piece<S>(a.out, row + p, o, a.out_cols - p, wide);
            }
        }
    }
}

template <class T, Store S, bool TWO>
__global__ __launch_bounds__(T::THREADS, T::FP * T::FQ > 32 ? 1 : 2)
void ffn_dx_kernel(FfnSum a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    ffn_sum_tile<T, S, true, TWO>(a, blockIdx.x, (SPH_LDS unsigned char*)smem_raw);
}

// dWg and dWu: `each` workgroups for the first, the rest for the second
template <class T, Store S, bool TWO>
__global__ __launch_bounds__(T::THREADS, T::FP * T::FQ > 32 ? 1 : 2)
void ffn_dw_kernel(FfnSum a, FfnSum b, int each)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    const bool second = (int)blockIdx.x >= each;
    ffn_sum_tile<T, S, false, TWO>(second ? b : a, (int)blockIdx.x - (second ? each : 0), (SPH_LDS unsigned char*)smem_raw);
}

// Slices added up in order, scaled and rounded, of up to three results: a wave 256 columns of a row, eight slices' loads under way
struct FfnJoin { FfnSum sum[3]; int columns[3]; long long until[2]; };   // waves below until[0] on the first, below until[1] on the second

template <Store S>
__global__ __launch_bounds__(256)
void ffn_join_kernel(FfnJoin j)
{
    const int lane = threadIdx.x & 63;
    const long long wave = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = wave < j.until[0] ? 0 : wave < j.until[1] ? 1 : 2;
    const FfnSum& a = j.sum[m];
    const int columns = max(j.columns[m], 1);
    const long long unit = wave - (m == 0 ? 0 : j.until[m - 1]), q = unit / columns;
    if (q >= a.out_rows) return;
    const int c = (int)(unit - q * columns) * 256 + lane * 4;
    if (c >= a.out_cols) return;
    const size_t slice = (size_t)a.out_rows * a.part_ld;
    const float* from = a.part + (size_t)q * a.part_ld + c;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 8;
    for (int s0 = 0; s0 < a.slices; s0 += AHEAD) {
        f32x4 y[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) y[i] = *(const f32x4*)(from + min(s0 + i, a.slices - 1) * slice);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (s0 + i < a.slices) x += y[i];
    }
    if constexpr (S == Store::F16) x *= a.row_down ? a.row_down[q] : 1.f;
    const size_t at = (size_t)q * a.out_ld + c;
    const int left = a.out_cols - c;
    if (left >= 4) {
        if constexpr (S == Store::F32) __builtin_memcpy((float*)a.out + at, &x, 16);
        else {
            const i32x2 w = {pack2<S == Store::F16>(x[0], x[1]), pack2<S == Store::F16>(x[2], x[3])};
            __builtin_memcpy((unsigned short*)a.out + at, &w, 8);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < left) store_el<S>(a.out, at + r, x[r]);
    }
}

// ---- around the products ------------------------------------------------------------------------------------

// X, Wg and Wu as the products take them (those with an `out`), and the norms of their rows (those with a `norm`): a wave per row.  Other types than fp16 take the squares' sum in
// fp64, whose range theirs do not leave.
struct FfnPack { PackRows m[3]; float* norm[3]; int until[2]; };   // workgroups below until[0] on the first, below until[1] on the second
constexpr int kFfnPackThreads = 256, kFfnPackRows = kFfnPackThreads / 64;

template <Store S>
__device__ __forceinline__ float row_norm(const PackRows& a, long long row, int lane)
{
    constexpr int N = per16<S>();
    const size_t from = (size_t)row * a.D, end = (size_t)a.n * a.D;
    const bool wide = ((uintptr_t)a.in & 15) == 0 && a.D % N == 0;
    std::conditional_t<S == Store::F16, float, double> sum = 0;
    for (int c = lane * N; c < a.D; c += 64 * N) {
        float x[N];
        widen16<S>(wide ? load16<S, true>(a.in, from + c, N, N) : load16<S, false>(a.in, from + c, a.D - c, end - from - c), x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (S == Store::F16) sum = __builtin_fmaf(x[i], x[i], sum);
            else sum = __builtin_fma((double)x[i], (double)x[i], sum);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if constexpr (S == Store::F16) return __builtin_sqrtf(sum);
    else return (float)__builtin_sqrt(sum);
}

template <Store S>
__global__ __launch_bounds__(kFfnPackThreads)
void ffn_pack_kernel(FfnPack a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), block = blockIdx.x;
    const int m = block < a.until[0] ? 0 : block < a.until[1] ? 1 : 2;
    const PackRows& rows = a.m[m];
    const long long row = (long long)(block - (m == 0 ? 0 : a.until[m - 1])) * kFfnPackRows + wave;
    if (row >= rows.n) return;
    if (a.norm[m]) {
        const float norm = row_norm<S>(rows, row, lane);
        if (lane == 0) a.norm[m][row] = norm;
    }
    pack_row<S>(rows, row, row, lane);
}

// fp16.  dA and dB are at most |dH| |x| |w| 1.13 for the rows' norms (act's slope is 1.13 at most), which a power of two brings to 2^13 .. 2^14: for dX by row t, of the largest
// |dH| of the row and the largest |w|; for dW, where dA and dB are a pair of their own, by column f, of the largest |dH| |x| of the column and its own |w| (one power for all of
// it lost the bits of units whose gradient is 2^-27 of that of others, as those of gates that are all but closed).  A dot product of D terms is about sqrt(D) below the product of
// the norms; from there down the type has 2^-14 for normal numbers, so with D = 2048 values keep their bits to 2^-22 of their row's or column's usual size.
// The largest |dH| of each row in each 512 columns, and the largest |dH| |x| of each column in each `rows` rows: a workgroup for both.  NaN counts for nothing, and neither does a row of X that is not finite.
constexpr int kTopCols = 512, kTopRows = 64, kTopMost = 64;   // (parts of a column at most)
template <bool EIGHT>                               // columns or more
__global__ __launch_bounds__(256)
void ffn_tops_kernel(const void* __restrict__ dH, const float* __restrict__ x_norm, int T, int F, int rows, float* __restrict__ row_top, float* __restrict__ col_top)
{
    constexpr Store S = Store::F16;
    constexpr int AHEAD = 16;                      // rows whose loads are under way
    __shared__ float shared[4][kTopCols];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = (F + kTopCols - 1) / kTopCols, tile = (int)(blockIdx.x % tiles), part = (int)(blockIdx.x / tiles);
    const int end = (int)min((long long)T, (long long)(part + 1) * rows);
    // (a row's last eight columns in the place of what goes past its end: the same maxima)
    const int c = min(tile * kTopCols + lane * 8, max(F - 8, 0));
    float col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) col[i] = 0.f;
    for (long long t0 = (long long)part * rows + wave * AHEAD; t0 < end; t0 += 4 * AHEAD) {
        const int last = min(AHEAD, (int)(end - t0)) - 1;      // (and the last row more than once)
        const unsigned short* const from = (const unsigned short*)dH + (size_t)t0 * F + c;
        i32x4 w[AHEAD];
        float norm[AHEAD], top[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int r = min(a, last);
            if constexpr (EIGHT) __builtin_memcpy(&w[a], from + (uint32_t)(r * F), 16);
            else w[a] = load16<S, false>(from, (size_t)r * F, F, (size_t)(T - t0 - r) * F);
            norm[a] = x_norm[t0 + r];
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            float x[8];
            widen16<S>(w[a], x);
            top[a] = 0.f;
            norm[a] = norm[a] < __builtin_inff() ? norm[a] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float size = __builtin_fabsf(x[i]);
                top[a] = fmaxf(top[a], size);
                col[i] = fmaxf(col[i], size * norm[a]);
            }
        }
        // sixteen maxima over the wave: half of the rows go to the lanes across at each exchange, in the end row r is with lanes 4 r .. 4 r + 3
        auto halve = [&](auto half) {
            constexpr int H = decltype(half)::value;
            const bool upper = (lane & 4 * H) != 0;
#pragma unroll
            for (int i = 0; i < H; ++i) {
                const float other = __shfl_xor(upper ? top[i] : top[i + H], 4 * H);
                top[i] = fmaxf(upper ? top[i + H] : top[i], other);
            }
        };
        static_assert(AHEAD == 16, "");
        halve(std::integral_constant<int, 8>{});
        halve(std::integral_constant<int, 4>{});
        halve(std::integral_constant<int, 2>{});
        halve(std::integral_constant<int, 1>{});
        top[0] = fmaxf(top[0], __shfl_xor(top[0], 2));
        top[0] = fmaxf(top[0], __shfl_xor(top[0], 1));
        if ((lane & 3) == 0 && t0 + (lane >> 2) < end) row_top[(size_t)tile * T + t0 + (lane >> 2)] = top[0];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) shared[wave][lane * 8 + i] = col[i];
    __syncthreads();
    for (int i = threadIdx.x; i < kTopCols; i += 256) {
        const int own = tile * kTopCols + i / 8 * 8, f = min(own, max(F - 8, 0)) + i % 8;   // (the column of this place; each is written by the lane that it belongs to)
        if (f >= own && f < F) col_top[(size_t)part * F + f] = fmaxf(fmaxf(shared[0][i], shared[1][i]), fmaxf(shared[2][i], shared[3][i]));
    }
}

// The rows' factors and the columns': a thread each, rows first.  One whose bound is infinite or 0 keeps its values as they are.
constexpr int kFactorThreads = 1024;
__global__ __launch_bounds__(kFactorThreads)
void ffn_factors_kernel(const float* __restrict__ x_norm, const float* __restrict__ w_norm, const float* __restrict__ row_top, const float* __restrict__ col_top, int T, int F, int parts,
                        float* __restrict__ row_up, float* __restrict__ row_down, int* __restrict__ col_up, float* __restrict__ down_a, float* __restrict__ down_b)
{
    __shared__ float shared[kFactorThreads / 64];
    const int tid = threadIdx.x;
    auto power = [](float x) { return x > 0.f && x < __builtin_inff() ? max(-100, min(100, 13 - (__builtin_amdgcn_frexp_expf(x) - 1))) : 0; };
    auto largest = [](const float* from, int n, int apart) {   // of every apart-th, eight loads under way
        float top = 0.f;
        for (int i0 = 0; i0 < n; i0 += 8) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = from[(size_t)min(i0 + i, n - 1) * apart];
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i]);
        }
        return top;
    };
    const long long unit = (long long)blockIdx.x * kFactorThreads + tid, f = unit - T;
    const float top = unit < T ? largest(row_top + unit, (F + kTopCols - 1) / kTopCols, T) : f < F ? largest(col_top + f, parts, F) : 0.f;
    float w = 0.f;                                 // (each workgroup for itself: a launch less)
#pragma unroll 4
    for (int i = tid; i < 2 * F; i += kFactorThreads) w = w_norm[i] < __builtin_inff() ? fmaxf(w, w_norm[i]) : w;
    w = max_over_wave(w);
    if ((tid & 63) == 0) shared[tid >> 6] = w;
    __syncthreads();
    for (int i = 0; i < kFactorThreads / 64; ++i) w = fmaxf(w, shared[i]);
    if (unit < T) {
        const int e = power(x_norm[unit] * top * w * 1.13f);
        row_up[unit] = __builtin_ldexpf(1.f, e);
        row_down[unit] = __builtin_ldexpf(1.f, -e);
    } else if (f < F) {
        const int a = power(top * w_norm[F + f] * 1.13f), b = power(top * w_norm[f] * 1.13f);
        col_up[f] = (a & 0xffff) | b << 16;
        down_a[f] = __builtin_ldexpf(1.f, -a);
        down_b[f] = __builtin_ldexpf(1.f, -b);
    }
}

}  // namespace sphattn
