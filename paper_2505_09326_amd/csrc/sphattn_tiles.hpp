// Products of matrices in tiles on the matrix instructions, and the parts that fp32 is multiplied in, for the kernels around the attention.
#pragma once
#include "sphattn_pipelined.hpp"
#include "sphattn_store.hpp"

namespace sphattn {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

constexpr float kLowPart = 4096.f;                 // what the second fp16 part is multiplied by: below 2^-14 that type has fewer bits
constexpr int kEndless = 1 << 20;                  // in place of the power of two of a row with an infinite element

// ---- tile products -------------------------------------------------------------------------------------

// out[q][p] = sum_k P[p][k] Q[q][k].  An operand is stored with rows along k ("across": row k holds all p) or with
// rows of k.  P's index lies along a lane's registers, Q's along the lanes.
struct Operand {
    const unsigned char* data;                     // 16-byte aligned
    long long part;                                // bytes from one part to the next (fp32)
    int ld;                                        // bytes per row, a multiple of 16
    int size;                                      // valid p or q (across: columns, a multiple of 8)
};

template <int BP_, int BQ_, int WAVES_P_, int WAVES_Q_, int NBUF_>
struct Tile {
    static constexpr int BP = BP_, BQ = BQ_, WAVES_P = WAVES_P_, WAVES_Q = WAVES_Q_, NBUF = NBUF_;
    static constexpr int WAVES = WAVES_P * WAVES_Q, THREADS = 64 * WAVES;
    static constexpr int FP = BP / WAVES_P / 16, FQ = BQ / WAVES_Q / 16;      // fragments of a wave
    // 1 KB copies per wave and step; where there are fewer blocks than waves several copy the same one (the same bytes)
    static constexpr int CP = BP / 16 / WAVES, CQ = (BQ / 16 + WAVES - 1) / WAVES, COPIES = CP + CQ;
    static constexpr int BUF = (BP + BQ) * 64, LDS = NBUF * BUF;
    static_assert(CP * WAVES * 16 == BP && (CQ * WAVES * 16 == BQ || CQ == 1), "");
};
constexpr int kStepK = 32;

// place of 16-byte piece c in row k of an operand stored across, and the piece in place c
__device__ __forceinline__ int across_slot(int k, int c) { return c ^ (2 * ((k & 3) | (k >> 1 & 4))); }

// Tiles of 256 x 256 on eight waves of 128 x 64: an operand byte in LDS feeds four or eight matrix instructions, 0.4 LDS reads per instruction (0.75
// transposed), and 128 KB of LDS hold four steps.
// The sum over k runs in steps of 32.  A step's part of the two operands is BP / 16 + BQ / 16 blocks of 1 KB, copied
// straight into one of NBUF LDS buffers, NBUF - 1 steps ahead; a step's fragments are read from LDS while the matrix
// instructions of the step before run, so that behind the one barrier per step the matrix pipe has its operands already.
//
// Beside one product there are two at once, P's and P2's rows with Q (Form::Two: a tile has BP / 2 of each, sixteen by sixteen in turn, so that fragments
// 2 i and 2 i + 1 of a wave are the same p of either), and the sum of two, P Q and P2 Q2 one after the other (Form::Sum).  P2 and Q2 are of P's and Q's sizes.
enum class Form { One, Two, Sum };

template <class T, bool HALF, bool PX, bool QX, int PAIRS, Form FORM = Form::One>
struct Product {
    f32x4 acc[T::FP][T::FQ];

    __device__ __forceinline__ void run(const Operand& P, const Operand& Q, int p0, int q0, int k0, int k_end,
                                        SPH_LDS unsigned char* smem, const Operand& P2 = Operand{}, const Operand& Q2 = Operand{})
    {
        static_assert(FORM != Form::Two || (!PX && T::CP % 2 == 0), "");
        static_assert(FORM != Form::Sum || PAIRS != 3, "");
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int n16 = lane & 15, g = lane >> 4;
        const int wp = wave % T::WAVES_P, wq = wave / T::WAVES_P;
        const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
        const int steps = (k_end - k0 + kStepK - 1) / kStepK;
        const int total = steps * PAIRS * (FORM == Form::Sum ? 2 : 1);

        // A copy's lane: rows of k lie in blocks of 16 x 64 bytes, lane l on row l / 4 with the piece of its slot.  Across, the buffer
        // holds 32 whole rows of the tile, so that a copy fetches whole lines of memory, their 16-byte pieces exchanged by
        // row (across_slot) so that the transposing reads of eight rows fall on different banks.
        const int row = lane >> 2, piece = block_piece_in_slot(lane);
        int voff[T::COPIES];
        uint32_t at[T::COPIES];                    // place in a buffer
        auto place = [&](bool across, const Operand& A, int a0, int size, int b, int& v) {
            if (!across) v = (b * 16 + row) * A.ld + piece * 16;
            else {
                const int slots = size / 8, k = (b * 64 + lane) / slots, col = a0 + across_slot(k, lane % slots) * 8;
                v = col < A.size ? k * A.ld + col * 2 : 0x7fffffff;
            }
        };
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) {
            const int b = i < T::CP ? wave * T::CP + i : (wave * T::CQ + (i - T::CP)) % (T::BQ / 16);
            place(i < T::CP ? PX : QX, i < T::CP ? P : Q, i < T::CP ? p0 : q0, i < T::CP ? T::BP : T::BQ, FORM == Form::Two && i < T::CP ? b / 2 : b, voff[i]);
            at[i] = (i < T::CP ? 0 : T::BP * 64) + b * 1024;
        }
        // where the next step's part begins, and (rows of k) how many bytes or (across) how many rows are left.  All of it in
        // scalar registers, which have no 64-bit comparisons.
        struct Stream { const unsigned char* base; int left; };
        auto start = [&](bool across, const Operand& A, int a0, int size, int part) {
            const int rows = min(size, A.size - a0);
            return across ? Stream{A.data + part * A.part + (long long)k0 * A.ld, k_end - k0}
                          : Stream{A.data + part * A.part + (long long)a0 * A.ld + (long long)k0 * 2, rows * A.ld - k0 * 2};
        };
        // parts of P and Q by pair, small products first: of Q's two (0,1) (0,0), of two of each (1,0) (0,1) (0,0), of three (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
        static_assert(PAIRS == 1 || PAIRS == 2 || PAIRS == 3 || PAIRS == 6, "");
        int pair = 0, step = 0, copied = 0;        // of the next copies
        auto part_p = [&]() { return PAIRS == 3 ? pair == 0 : PAIRS == 6 ? (pair == 0 ? 2 : pair == 2 || pair == 3) : 0; };
        auto part_q = [&]() { return PAIRS == 2 ? pair == 0 : PAIRS == 3 ? pair == 1 : PAIRS == 6 ? (pair == 1 ? 2 : pair == 2 || pair == 4) : 0; };
        constexpr int ROWS_P = FORM == Form::Two ? T::BP / 2 : T::BP;
        Stream sp = start(PX, P, p0, ROWS_P, part_p()), sq = start(QX, Q, q0, T::BQ, part_q());
        Stream sp2 = FORM == Form::Two ? start(PX, P2, p0, ROWS_P, part_p()) : sp;
        bool second = false;                       // Form::Sum: of the second product
        uint32_t to = lds0;
        auto words = [&](bool across, const Operand& A, const Stream& s, bool there) {
            const int left = there ? max(s.left, 0) : 0;
            return rsrc_words(s.base, (uint32_t)__builtin_amdgcn_readfirstlane(across ? min(left, kStepK) * A.ld : left));
        };
        // of the step that is copied next
        i32x4 rp, rq, rp2;
        bool past = false;
        auto copy_begin = [&]() {
            const bool there = copied < total;
            rp = words(PX, P, sp, there);
            if constexpr (FORM == Form::Two) rp2 = words(PX, P2, sp2, there);
            rq = words(QX, Q, sq, there);
            past = k0 * 2 + step * 64 + piece * 16 >= k_end * 2;   // pieces behind the end of the sum are zeros
        };
        auto copy_one = [&](int i) {
            const bool across = i < T::CP ? PX : QX;
            copy_to_lds(i >= T::CP ? rq : FORM == Form::Two && i % 2 ? rp2 : rp, to + at[i], !across && past ? 0x7fffffff : voff[i], 0);
        };
        auto copy_end = [&]() {
            ++copied;
            ++step;
            to = to == lds0 + (T::NBUF - 1) * T::BUF ? lds0 : to + T::BUF;
            sp.base += PX ? (long long)kStepK * P.ld : 64;
            sp.left -= PX ? kStepK : 64;
            sq.base += QX ? (long long)kStepK * Q.ld : 64;
            sq.left -= QX ? kStepK : 64;
            if constexpr (FORM == Form::Two) {
                sp2.base += 64;
                sp2.left -= 64;
            }
            if ((PAIRS > 1 || FORM == Form::Sum) && step == steps && copied < total) {
                step = 0;
                ++pair;
                if (FORM == Form::Sum && pair == PAIRS) second = true, pair = 0;
                sp = start(PX, FORM == Form::Sum && second ? P2 : P, p0, ROWS_P, part_p());
                sq = start(QX, FORM == Form::Sum && second ? Q2 : Q, q0, T::BQ, part_q());
                if constexpr (FORM == Form::Two) sp2 = start(PX, P2, p0, ROWS_P, part_p());
            }
        };
        auto copy_step = [&]() {
            copy_begin();
#pragma unroll
            for (int i = 0; i < T::COPIES; ++i) copy_one(i);
            copy_end();
        };

        i32x4 pf[T::FP], qf[2][T::FQ];
        auto fragment = [&](bool across, const SPH_LDS unsigned char* block0, int size, int i) -> i32x4 {
            if (!across) return lds_read_b128(block0 + i * 1024 + block_piece_offset(n16, g));
            // lane (i, g): rows 8 g + i / 4 and 4 more, columns 4 (i % 4) .. + 3 of the sixteen
            const int k = 8 * g + (n16 >> 2), at = across_slot(k, 2 * i + ((lane >> 1) & 1)) * 16 + (lane & 1) * 8;
            const SPH_LDS unsigned char* b = block0 + k * size * 2 + at;
            const i32x2 lo = lds_read_tr64(b), hi = lds_read_tr64(b + 4 * size * 2);   // (rows k and k + 4 exchange alike)
            return i32x4{lo[0], lo[1], hi[0], hi[1]};
        };
        auto read_p = [&](uint32_t from, int i) {
            pf[i] = fragment(PX, smem + from + (PX ? 0 : wp * T::FP * 1024), T::BP, PX ? wp * T::FP + i : i);
        };
        auto read_q = [&](uint32_t from, int set, int j) {
            qf[set][j] = fragment(QX, smem + from + T::BP * 64 + (QX ? 0 : wq * T::FQ * 1024), T::BQ, QX ? wq * T::FQ + j : j);
        };
        auto behind = [](uint32_t from) { return from == (T::NBUF - 1) * T::BUF ? 0u : from + T::BUF; };
        constexpr int VM = (T::NBUF - 3) * T::COPIES;   // copies that may still be under way when the next step's have to be there
        static_assert(T::NBUF >= 3 && VM < 64, "");
        auto arrive = [&]() {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0x0F70 | (VM & 15) | ((VM >> 4) << 14));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };

#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int j = 0; j < T::FQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // (every step is copied, those past the last one as zeros, which add nothing: the loop takes two at a time)
#pragma unroll
        for (int s = 0; s < T::NBUF - 2; ++s) copy_step();
        copy_step();
        {
            constexpr int VM0 = (T::NBUF - 2) * T::COPIES;
            static_assert(VM0 < 64, "");
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0x0F70 | (VM0 & 15) | ((VM0 >> 4) << 14));
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
        uint32_t from = 0;                         // buffer of step s
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) read_q(from, 0, j);
#pragma unroll
        for (int i = 0; i < T::FP - 1; ++i) read_p(from, i);
        for (int s = 0; s < total; s += 2) {
            // of three products the first two have a second part, 2^12 times as large as it is: an even number of steps, after which the sums are brought back
            if (PAIRS == 3 && s == 2 * steps) {
#pragma unroll
                for (int i = 0; i < T::FP; ++i)
#pragma unroll
                    for (int j = 0; j < T::FQ; ++j) acc[i][j] *= 1.f / kLowPart;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                arrive();                          // step s + u + 1 is there; the fragments of step s + u - 1 are used up
                copy_begin();                      // into that one's buffer
                const uint32_t next = behind(from);
                // One P fragment with all of Q at a time, and beside these products a share of the step's copies and of the reads for the
                // next one.  All copies behind the barrier would queue at the memory pipe, eight waves' at once, and the products
                // behind them in the program with them; left to itself the compiler also puts a read right before the product that
                // needs it.  A P fragment is used up when its products are done and makes place for the next step's (the last
                // one's place is taken a step later); Q's are needed to the end and have two sets.
#pragma unroll
                for (int i = 0; i < T::FP; ++i) {
#pragma unroll
                    for (int c = i * T::COPIES / T::FP; c < (i + 1) * T::COPIES / T::FP; ++c) copy_one(c);
                    if (i == 0) read_p(from, T::FP - 1);
                    else read_p(next, i - 1);
                    const int q0f = i * T::FQ / T::FP, q1f = (i + 1) * T::FQ / T::FP;
#pragma unroll
                    for (int j = q0f; j < q1f; ++j) read_q(next, u ^ 1, j);
#pragma unroll
                    for (int j = 0; j < T::FQ; ++j) {   // to and fro: one operand changes at a time
                        const int jj = i & 1 ? T::FQ - 1 - j : j;
                        acc[i][jj] = mfma16x16<HALF>(pf[i], qf[u][jj], acc[i][jj]);
                    }
                    const int reads = (PX ? 2 : 1) + (q1f - q0f) * (QX ? 2 : 1);
#pragma unroll
                    for (int j = 0; j < T::FQ; ++j) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                        if (j < reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                copy_end();
                from = next;
            }
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);        // vmcnt(0), lgkmcnt(0): nothing of this lands in what follows
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
};

// Workgroup -> tile.  Each XCD takes a contiguous range; within it, groups of eight q tiles are walked p by p, so that the
// workgroups that run together share operand panels in the XCD's L2.
struct TileAt { int p, q, slice; };
__device__ __forceinline__ TileAt tile_of(int id, int tiles_p, int tiles_q)
{
    constexpr int GROUP = 8;
    const int per_slice = tiles_p * tiles_q, slice = id / per_slice;
    id -= slice * per_slice;
    const int per_group = GROUP * tiles_p, group = id / per_group, in = id - group * per_group;
    const int rows = min(GROUP, tiles_q - group * GROUP);
    return TileAt{in / rows, group * GROUP + in % rows, slice};
}

// ---- parts of fp32 -----------------------------------------------------------------------------------------

// A value (2^15 at most) as two fp16 parts.  NaN: in the first.
__device__ __forceinline__ void split2(float x, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)x;
    lo = (_Float16)((x - (float)hi) * kLowPart);
    if (__builtin_fabsf(x) == __builtin_inff() || x != x) lo = (_Float16)0.f;
}

// Four neighbouring values' parts
__device__ __forceinline__ void split2(const float (&x)[4], i32x2& hi, i32x2& lo)
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        _Float16 a, b, c, d;
        split2(x[2 * r], a, b);
        split2(x[2 * r + 1], c, d);
        hi[r] = __builtin_bit_cast(int, f16x2{a, c});
        lo[r] = __builtin_bit_cast(int, f16x2{b, d});
    }
}

// Four neighbouring values as three bf16 parts that are them (8 + 8 + 8 bits), over the whole range of fp32.  Infinite or NaN: in the first.
__device__ __forceinline__ void split3(const float (&x)[4], i32x2 (&part)[3])
{
    constexpr float MOST = 0x1.fep127f;            // (a finite value is not to be rounded to an infinite one)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float left[2];
        bool finite[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            left[i] = x[2 * r + i];
            finite[i] = __builtin_fabsf(left[i]) < __builtin_inff();
        }
        const int hi = pack2<false>(finite[0] ? fminf(fmaxf(left[0], -MOST), MOST) : left[0], finite[1] ? fminf(fmaxf(left[1], -MOST), MOST) : left[1]);
        left[0] = finite[0] ? left[0] - __builtin_bit_cast(float, hi << 16) : 0.f;
        left[1] = finite[1] ? left[1] - __builtin_bit_cast(float, hi & (int)0xffff0000) : 0.f;
        const int mid = pack2<false>(left[0], left[1]);
        part[0][r] = hi;
        part[1][r] = mid;
        part[2][r] = pack2<false>(left[0] - __builtin_bit_cast(float, mid << 16), left[1] - __builtin_bit_cast(float, mid & (int)0xffff0000));
    }
}

// Two accumulator fragments' rows of four 16-bit values, lane group g holding columns 4 g .. 4 g + 3 of each: afterwards group g has
// columns 8 (g / 2) .. + 7 of fragment g % 2.
__device__ __forceinline__ i32x4 join_fragments(i32x2 a, i32x2 b)
{
    int a0 = a[0], a1 = a[1], b0 = b[0], b1 = b[1];
    // (odd rows of sixteen lanes of the first operand and even rows of the second change places)
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %2\n\tv_permlane16_swap_b32 %1, %3\n\ts_nop 1" : "+v"(a0), "+v"(a1), "+v"(b0), "+v"(b1));
    return i32x4{a0, a1, b0, b1};
}

// What two values' rounding to the 16-bit type has left of them, rounded (of what is not finite there: nothing)
template <bool HALF>
__device__ __forceinline__ int pack2_rest(float a, float b, int rounded)
{
    float x, y;
    if constexpr (HALF) {
        const f16x2 h = __builtin_bit_cast(f16x2, rounded);
        x = (float)h[0], y = (float)h[1];
    } else {
        x = __builtin_bit_cast(float, rounded << 16), y = __builtin_bit_cast(float, rounded & (int)0xffff0000);
    }
    return pack2<HALF>(__builtin_fabsf(x) < __builtin_inff() ? a - x : 0.f, __builtin_fabsf(y) < __builtin_inff() ? b - y : 0.f);
}

// D = A (16 x 4) B (4 x 16) + C on element ea of a's registers and eb of b's
__device__ __forceinline__ f32x4 mfma_f32(i32x4 a, int ea, i32x4 b, int eb, f32x4 c)
{
    const int x = a[ea], y = b[eb];                // (a bit cast of the vector's element itself takes the vector's first)
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(i32x4 a, i32x4 b, int e, f32x4 c) { return mfma_f32(a, e, b, e, c); }

__device__ __forceinline__ float max_over_wave(float x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// Rows as the products want them: 16-bit, 16-byte aligned, whole pieces of 8; fp32 in parts.  One wave per row.
struct PackRows {
    const void* in; void* out; int n, D, ld;       // (ld: elements per row of out, a multiple of 8)
    long long part;                                // elements from part to part
    void* sum_out;                                 // fp32: the three parts that the products with G take, or NULL
    int* exp;                                      // fp32: for the logits, the power of two that the row was divided by
};
template <Store S>
__device__ __forceinline__ void pack_row(const PackRows& a, long long t, long long m, int lane)
{
    if (!a.out) return;                            // (few rows of fp32 are read where they are)
    const size_t from = (size_t)t * a.D, to = (size_t)m * a.ld;
    constexpr int N = per16<S>();
    const bool wide = ((uintptr_t)a.in & 15) == 0 && a.D % N == 0;
    auto load = [&](int c) { return wide ? load16<S, true>(a.in, from + c, N, N) : load16<S, false>(a.in, from + c, a.D - c, (size_t)a.n * a.D - from - c); };
    int up = 0;
    if constexpr (S == Store::F32) {               // the row's largest finite element goes to 2^14 .. 2^15
        float top = 0.f;
        bool endless = false;
        for (int c = lane * N; c < a.D; c += 64 * N) {
            float x[N];
            widen16<S>(load(c), x);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float size = __builtin_fabsf(x[i]);
                top = size < __builtin_inff() ? fmaxf(top, size) : top;
                endless |= size == __builtin_inff();
            }
        }
        top = max_over_wave(top);
        up = top > 0.f ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
        if (__ballot(endless) && lane == 0) a.exp[m] = kEndless;
        else if (lane == 0) a.exp[m] = -up;
    }
    for (int c = lane * N; c < a.ld; c += 64 * N) {
        i32x4 w = {0, 0, 0, 0};
        if (c < a.D) w = load(c);
        if constexpr (S == Store::F32) {
            float x[4];
            widen16<S>(w, x);
            i32x2 hi, lo;
            if (a.sum_out) {
                i32x2 part[3];
                split3(x, part);
#pragma unroll
                for (int k = 0; k < 3; ++k) *(i32x2*)((unsigned short*)a.sum_out + to + c + k * a.part) = part[k];
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = __builtin_ldexpf(x[r], up);
            split2(x, hi, lo);
            unsigned short* o = (unsigned short*)a.out + to + c;
            *(i32x2*)o = hi;
            *(i32x2*)(o + a.part) = lo;
        } else {
            *(i32x4*)((unsigned short*)a.out + to + c) = w;
        }
    }
}

}  // namespace sphattn
