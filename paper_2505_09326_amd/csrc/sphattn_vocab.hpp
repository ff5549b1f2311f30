// Cross entropy over a large vocabulary without keeping the logits, and its gradients, for gfx950.
//
//   l_tv = c x_t . w_v      lse_t = log sum_v exp l_tv      loss_t = lse_t - l_{t,y_t}
//   G_tv = g_t (exp(l_tv - lse_t) - [v = y_t])      dX = c G W      dW = c G^T X
// (one g for all rows and c are applied to the sums instead)
//
// Three kinds of matrix product run on one tile kernel:
//   logits   each tile of T x V is reduced, in registers, to a maximum and a sum of exponentials per row
//   G        the same tiles again for a piece of the vocabulary, each turned into 16-bit values of G in a workspace
//   dX, dW   products of that piece with W and X, the operand whose rows run along the sum read from LDS transposed
// The logits are formed twice (8 T V D operations for a training step instead of 6): a tile costs less than
// writing it as fp32 and reading it back.  G is rounded to the storage type, which is what the matrix instructions take (once, by 2^-8 of a term in bf16 and 2^-11
// in fp16 at most; that is a tenth of the whole error against 64 bits, most of which is the rounding of the results: 1.8e-3 against 1.7e-3 with G in fp32),
// sums are in fp32 throughout.
//
// Bound by the matrix pipes where the sums are long: 8192 rows, 65536 ids, width 2048 in bf16 7.0 to 7.2 ms, 8 T V D at 1226 to 1257 TFLOP/s, what a
// library product of 8192^3 reaches (1266).  At width 1024 a tile's end, its exponentials and stores, has no other tile's products beside it: logits and
// G run at 0.57 busy pipes against 0.75 of dW (8192 x 32768 1.96 to 1.98 ms).  One row: W at 5.3 TB/s.
//
// fp32 storage, logits: X and W are written as two fp16 parts each, the value rounded and 2^12 times what that left out rounded (11 + 11 bits, of
// the value times a power of two that brings its row's largest element to 2^14 .. 2^15), and a product is three
// products of parts, the small ones first, on the same kernel.  A factor is off by 2^-23 on average and 2^-22 at most, below 2^-29 of its
// row's largest element by 2^-51 of that; the product left out comes to 2^-22 of a term at most.  The powers of two come back to the logits in a tile's end,
// so no row takes bits from another (one for all of W lost every id beside a bias of -1e9).  Rows with an infinite element, which a product of parts makes
// NaN of where the other part is zero, take fp32 products there instead.
// Gradients: G, X and W as three bf16 parts each, which are the value over the whole range of fp32, and six products; what is left out comes to 2^-24 of
// a term.  (Two fp16 parts and three products took 273 us for 1999 x 8000 x 512 where this takes 394 to 412, but hold nothing below 2^-39 of the
// largest: a row of dX whose gradient is 1e-8 of another's lost 2 % of itself, ids that no row gives a weight above 1e-12 their whole row of dW.)
// Up to 64 rows, where reading W is most of the time, use fp32 matrix instructions on fp32 as it is: RowsProduct.
#pragma once
#include "sphattn_embed.hpp"
#include "sphattn_pipelined.hpp"

#include <type_traits>

namespace sphattn {

// What the host cannot know: how many rows count, and how their gradients are scaled.
struct VocabInfo {
    int rows;                                      // rows with a target
    float up;                                      // factor of G in the workspace: a power of two (fp16 holds G near 2^14 with it)
    float down;                                    // factor of the sums behind it
    int even;                                      // one gradient per row, fp16: all of them within 2^4 of the largest, so that one `up` serves every row
};

constexpr float kLowPart = 4096.f;                 // what the second fp16 part is multiplied by: below 2^-14 that type has fewer bits
constexpr int kEndless = 1 << 20;                  // in place of the power of two of a row with an infinite element

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

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
template <class T, bool HALF, bool PX, bool QX, int PAIRS>
struct Product {
    f32x4 acc[T::FP][T::FQ];

    __device__ __forceinline__ void run(const Operand& P, const Operand& Q, int p0, int q0, int k0, int k_end,
                                        SPH_LDS unsigned char* smem)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int n16 = lane & 15, g = lane >> 4;
        const int wp = wave % T::WAVES_P, wq = wave / T::WAVES_P;
        const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
        const int steps = (k_end - k0 + kStepK - 1) / kStepK;
        const int total = steps * PAIRS;

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
            place(i < T::CP ? PX : QX, i < T::CP ? P : Q, i < T::CP ? p0 : q0, i < T::CP ? T::BP : T::BQ, b, voff[i]);
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
        // parts of P and Q by pair, small products first: (1,0) (0,1) (0,0), or of three parts (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
        static_assert(PAIRS == 1 || PAIRS == 3 || PAIRS == 6, "");
        int pair = 0, step = 0, copied = 0;        // of the next copies
        auto part_p = [&]() { return PAIRS == 3 ? pair == 0 : PAIRS == 6 ? (pair == 0 ? 2 : pair == 2 || pair == 3) : 0; };
        auto part_q = [&]() { return PAIRS == 3 ? pair == 1 : PAIRS == 6 ? (pair == 1 ? 2 : pair == 2 || pair == 4) : 0; };
        Stream sp = start(PX, P, p0, T::BP, part_p()), sq = start(QX, Q, q0, T::BQ, part_q());
        uint32_t to = lds0;
        auto words = [&](bool across, const Operand& A, const Stream& s, bool there) {
            const int left = there ? max(s.left, 0) : 0;
            return rsrc_words(s.base, (uint32_t)__builtin_amdgcn_readfirstlane(across ? min(left, kStepK) * A.ld : left));
        };
        // of the step that is copied next
        i32x4 rp, rq;
        bool past = false;
        auto copy_begin = [&]() {
            const bool there = copied < total;
            rp = words(PX, P, sp, there);
            rq = words(QX, Q, sq, there);
            past = k0 * 2 + step * 64 + piece * 16 >= k_end * 2;   // pieces behind the end of the sum are zeros
        };
        auto copy_one = [&](int i) {
            const bool across = i < T::CP ? PX : QX;
            copy_to_lds(i < T::CP ? rp : rq, to + at[i], !across && past ? 0x7fffffff : voff[i], 0);
        };
        auto copy_end = [&]() {
            ++copied;
            ++step;
            to = to == lds0 + (T::NBUF - 1) * T::BUF ? lds0 : to + T::BUF;
            sp.base += PX ? (long long)kStepK * P.ld : 64;
            sp.left -= PX ? kStepK : 64;
            sq.base += QX ? (long long)kStepK * Q.ld : 64;
            sq.left -= QX ? kStepK : 64;
            if (PAIRS > 1 && step == steps && copied < total) {
                step = 0;
                ++pair;
                sp = start(PX, P, p0, T::BP, part_p());
                sq = start(QX, Q, q0, T::BQ, part_q());
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

struct VocabArgs {
    Operand P, Q;
    const VocabInfo* info;                         // NULL: all rows of Q count
    // fp32 in parts: the powers of two that each row was divided by (or kEndless), and the rows as they are
    const int *p_exp, *q_exp; const float *p_whole, *q_whole; int D;
    int k;                                         // length of the sum (dW: the rows that count)
    int first;                                     // tile of the launch's first workgroup
    int tiles_p, slices;
    int T, target;                                 // rows of X; dX: workgroups that the chip runs at once (0: slices are as they are)
    // logits and G: the vocabulary ids p0 .. of this launch, V of them in all
    int V, v0;
    float scale2;                                  // c log2(e)
    const void* targets; int id_bytes; const int* rows;   // targets[rows[q]], or targets[q] without rows
    float2* partial; int partial_ld; float* target_logit; // logits
    const int* g_target; const float* g_lse2; const float* g;   // G, by row that counts
    int unless_even;                               // G: already there if the rows' gradients are even
    void* G; long long G_part; int G_ld;           // (elements)
    // dX, dW
    void* out; int out_ld; int out_cols, out_rows; int accumulate;   // (dX: slice after slice, `rows` rows each)
};

enum class Stage { Logits, G, Dx, Dw };

// Slices of dX's sum over the vocabulary for `rows` rows that count, where a launch for T of them has `slices`: as many more as
// workgroups and arrays of partial sums are then free, while the chip is not full.  (8000 rows of which 1200 count, 20011 ids, width 1024:
// dX 169 -> 56 us, and 15 to add the slices up where it was 6.)
__device__ __forceinline__ int dx_slices(int rows, int T, int slices, int tile_q, int tiles_p, int target)
{
    const int tq = (rows + tile_q - 1) / tile_q, tq_all = (T + tile_q - 1) / tile_q;
    if (rows <= 0) return slices;
    const int room = (int)min((long long)tq_all * slices / tq, (long long)T * slices / rows);
    return max(slices, min(min(room, 32), target / (tq * tiles_p)));
}

// D = A (16 x 4) B (4 x 16) + C on element ea of a's registers and eb of b's
__device__ __forceinline__ f32x4 mfma_f32(i32x4 a, int ea, i32x4 b, int eb, f32x4 c)
{
    const int x = a[ea], y = b[eb];                // (a bit cast of the vector's element itself takes the vector's first)
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(i32x4 a, i32x4 b, int e, f32x4 c) { return mfma_f32(a, e, b, e, c); }

// fp32 with at most 64 rows: W decides the time, so it is read as it is, once, straight into registers, and multiplied by the fp32 matrix
// instruction (16x16x4, a twelfth of the 16-bit rate: 64 rows of width 1024 take it as long as their W takes memory).  Lane (i, g) holds four neighbouring
// k, 4 g .. 4 g + 3 of sixteen, of row i of both operands, and instruction r takes the r-th: any order of k will do if both have it.
// (17 rows, 50000 x 1024: logits 68 us, W at 3.0 TB/s, dX 57, dW 62, a training step 277; with parts in memory 489.  64 rows, 60000 x 1472: 165, 149, 179,
// and 655 against 840, which the instruction's rate is less than half of: X's fragments are loaded in the step that multiplies them.  3 rows, 20000 x
// 512: 17.6, 11, 12.)
template <class T>
struct RowsProduct {
    f32x4 acc[T::FP][T::FQ];

    __device__ __forceinline__ void run(const VocabArgs& a, int rows, int p0, int q0)
    {
        constexpr int CH = T::FQ > 1 ? 2 : 4;      // times sixteen k under way, and as many being multiplied
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4, D = a.k;
        const float *W = (const float*)a.P.data, *X = (const float*)a.Q.data;
        const bool wide = (((uintptr_t)W | (uintptr_t)X) & 15) == 0 && D % 4 == 0;
        size_t pat[T::FP], qat[T::FQ];             // (rows behind the last one take the last one's place: their results are not looked at)
#pragma unroll
        for (int i = 0; i < T::FP; ++i) pat[i] = (size_t)min(p0 + (wave * T::FP + i) * 16 + n16, a.P.size - 1) * D;
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) {
            const int q = min(q0 + j * 16 + n16, rows - 1);
            qat[j] = (size_t)(a.rows ? a.rows[q] : q) * D;
        }
        auto load = [&](const float* from, size_t at, int k, size_t all) {
            if (k >= D) return i32x4{0, 0, 0, 0};
            return wide ? load16<Store::F32, true>(from, at + k, 4, 4) : load16<Store::F32, false>(from, at + k, D - k, all - at - k);
        };
        i32x4 next[CH][T::FP];
        auto fetch = [&](int k) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < T::FP; ++i) next[c][i] = load(W, pat[i], k + 16 * c + 4 * g, (size_t)a.P.size * D);
        };
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int j = 0; j < T::FQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        fetch(0);
        for (int k = 0; k < D; k += 16 * CH) {
            i32x4 w[CH][T::FP], x[CH][T::FQ];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
#pragma unroll
                for (int i = 0; i < T::FP; ++i) w[c][i] = next[c][i];
#pragma unroll
                for (int j = 0; j < T::FQ; ++j) x[c][j] = load(X, qat[j], k + 16 * c + 4 * g, (size_t)a.T * D);
            }
            fetch(k + 16 * CH);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < T::FP; ++i)
#pragma unroll
                        for (int j = 0; j < T::FQ; ++j) acc[i][j] = mfma_f32(w[c][i], x[c][j], r, acc[i][j]);
        }
    }
};

// dX of those: G [rows, n] in fp32 times W, a wave 64 columns and a slice of the ids.  Lane (i, g) reads four neighbouring columns 4 i of ids
// 4 g + r, so that each of them is a fragment of its own and a row's 64 columns leave as 256 bytes.
template <int FT>
__global__ __launch_bounds__(256)
void vocab_rows_dx_kernel(VocabArgs a)
{
    constexpr int CH = 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int rows = a.info->rows, D = a.k, n = a.P.size, blocks = (D + 63) / 64;
    const int unit = (int)blockIdx.x * 4 + wave, slice = unit / blocks, d = unit % blocks * 64 + 4 * n16, left = D - d;
    if (rows == 0 || slice >= a.slices) return;
    const int per = ((n + a.slices - 1) / a.slices + 15) / 16 * 16;
    const int v0 = (int)min((long long)n, (long long)slice * per), v1 = min(n, v0 + per);
    const float *W = (const float*)a.P.data, *G = (const float*)a.G;
    const bool wide = ((uintptr_t)W & 15) == 0 && D % 4 == 0;
    size_t gat[FT];
#pragma unroll
    for (int j = 0; j < FT; ++j) gat[j] = (size_t)min(j * 16 + n16, rows - 1) * a.G_ld;
    f32x4 acc[FT][4];
#pragma unroll
    for (int j = 0; j < FT; ++j)
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[j][f] = f32x4{0.f, 0.f, 0.f, 0.f};
    i32x4 next_w[CH][4], next_g[CH][FT];
    auto fetch = [&](int v) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = v + 16 * c + 4 * g;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const size_t from = (size_t)(at + r) * D + d;
                next_w[c][r] = i32x4{0, 0, 0, 0};
                if (at + r < v1 && left > 0) next_w[c][r] = wide ? load16<Store::F32, true>(W, from, 4, 4) : load16<Store::F32, false>(W, from, left, (size_t)n * D - from);
            }
#pragma unroll
            for (int j = 0; j < FT; ++j) {         // (columns from n on are zeros in G, up to a tile's end)
                next_g[c][j] = i32x4{0, 0, 0, 0};
                if (at < v1) next_g[c][j] = *(const i32x4*)(G + gat[j] + at);
            }
        }
    };
    fetch(v0);
    for (int v = v0; v < v1; v += 16 * CH) {
        i32x4 w[CH][4], x[CH][FT];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int r = 0; r < 4; ++r) w[c][r] = next_w[c][r];
#pragma unroll
            for (int j = 0; j < FT; ++j) x[c][j] = next_g[c][j];
        }
        fetch(v + 16 * CH);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < FT; ++j)
#pragma unroll
                    for (int f = 0; f < 4; ++f) acc[j][f] = mfma_f32(x[c][j], r, w[c][r], f, acc[j][f]);
    }
    if (left <= 0) return;
#pragma unroll
    for (int j = 0; j < FT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * j + 4 * g + r;
            if (t >= rows) continue;
            f32x4* to = (f32x4*)((float*)a.out + ((size_t)slice * rows + t) * a.out_ld + d);
            f32x4 o = {acc[j][0][r], acc[j][1][r], acc[j][2][r], acc[j][3][r]};
            if (a.accumulate) o += *to;
            *to = o;
        }
}

// dW of those: a wave 64 ids x 64 columns, sums over the rows that count.  X is read in place (rows[q]) and nothing
// ahead, so dW leaves at less than memory's rate: 17 rows, 50000 x 1024 at 3.3 TB/s, 64 rows, 60000 x 1472 at 2.0.
__global__ __launch_bounds__(256)
void vocab_rows_dw_kernel(VocabArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int rows = a.info->rows, D = a.k, n = a.out_rows, blocks = (D + 63) / 64;
    const float down = a.info->down;
    const long long unit = (long long)blockIdx.x * 4 + wave;
    const int v0 = (int)(unit / blocks) * 64, d = (int)(unit % blocks) * 64 + 4 * n16, left = D - d;
    if (v0 >= n) return;
    const float *X = (const float*)a.Q.data, *G = (const float*)a.G;
    const bool wide = (((uintptr_t)X | (uintptr_t)a.out) & 15) == 0 && D % 4 == 0;
    f32x4 acc[4][4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int f = 0; f < 4; ++f) acc[e][f] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < rows; t0 += 16) {
        i32x4 y[4], x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = t0 + 4 * g + r;
            y[r] = x[r] = i32x4{0, 0, 0, 0};
            if (t < rows) {
                y[r] = *(const i32x4*)(G + (size_t)t * a.G_ld + v0 + 4 * n16);
                const size_t at = (size_t)a.rows[t] * D + d;
                if (left > 0) x[r] = wide ? load16<Store::F32, true>(X, at, 4, 4) : load16<Store::F32, false>(X, at, left, (size_t)a.T * D - at);
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int f = 0; f < 4; ++f) acc[e][f] = mfma_f32(y[r], e, x[r], f, acc[e][f]);
    }
    if (left <= 0) return;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int v = v0 + 16 * g + 4 * r + e;
            if (v >= n) continue;
            const f32x4 o = f32x4{acc[e][0][r], acc[e][1][r], acc[e][2][r], acc[e][3][r]} * down;
            const size_t at = (size_t)v * D + d;
            if (wide) store16<Store::F32, true>(a.out, at, __builtin_bit_cast(i32x4, o), 4);
            else store16<Store::F32, false>(a.out, at, __builtin_bit_cast(i32x4, o), left);
        }
}

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

// whether logits and G are formed from fp32 as it is (RowsProduct)
template <class T, Store S, Stage ST>
constexpr bool reads_fp32() { return S == Store::F32 && T::BQ <= 64 && (ST == Stage::Logits || ST == Stage::G); }

// The logits of a wave's corner from rows of fp32 as they are, four k at a time: for the rare tile that meets a row with an infinite element, where only
// the formula itself says which infinity it is or that it is none.  Waits for nothing but its own loads.
template <class T>
__device__ __forceinline__ void whole_logits(f32x4 (&acc)[T::FP][T::FQ], const VocabArgs& a, int rows, int pw, int qw)
{
    const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
    const float *pat[T::FP], *qat[T::FQ];          // (rows behind the last one: see RowsProduct)
#pragma unroll
    for (int i = 0; i < T::FP; ++i) pat[i] = a.p_whole + (size_t)min(pw + 16 * i + n16, a.P.size - 1) * a.D;
#pragma unroll
    for (int j = 0; j < T::FQ; ++j) {
        const int q = min(qw + 16 * j + n16, rows - 1);
        qat[j] = a.q_whole + (size_t)(a.rows ? a.rows[q] : q) * a.D;
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

template <class T, Store S, Stage ST>
__device__ __forceinline__ void vocab_tile(const VocabArgs& a, int block, SPH_LDS unsigned char* smem)
{
    constexpr bool PX = ST == Stage::Dx || ST == Stage::Dw, QX = ST == Stage::Dw;
    int rows = a.Q.size, k = a.k;
    float down = 1.f;
    if (a.info) {
        rows = __builtin_amdgcn_readfirstlane(a.info->rows);
        if constexpr (ST == Stage::G && S == Store::F16)
            if (a.unless_even && __builtin_amdgcn_readfirstlane(a.info->even)) return;
        if constexpr (ST == Stage::Dw) down = a.info->down;
    }
    Operand Q = a.Q;
    if constexpr (ST == Stage::Dw) {
        k = rows;
        rows = a.Q.size;
    } else {
        Q.size = rows;
    }
    const int slices = ST == Stage::Dx ? __builtin_amdgcn_readfirstlane(dx_slices(rows, a.T, a.slices, T::BQ, a.tiles_p, a.target)) : 1;
    const int tiles_q = (rows + T::BQ - 1) / T::BQ, n_tiles = a.tiles_p * tiles_q * slices;
    const int id = block + a.first;
    if (id >= n_tiles) return;
    const TileAt tile = tile_of(xcd_contiguous_id(id, n_tiles), a.tiles_p, tiles_q);
    // (divisions leave their results in vector registers)
    const int p0 = __builtin_amdgcn_readfirstlane(tile.p) * T::BP, q0 = __builtin_amdgcn_readfirstlane(tile.q) * T::BQ;
    const int per_slice = __builtin_amdgcn_readfirstlane(((k + kStepK - 1) / kStepK + slices - 1) / slices) * kStepK;
    const int k0 = min(k, __builtin_amdgcn_readfirstlane(tile.slice) * per_slice), k1 = min(k, k0 + per_slice);

    constexpr bool ROWS = reads_fp32<T, S, ST>();
    constexpr bool SUMS = ST == Stage::Dx || ST == Stage::Dw, F32 = S == Store::F32;
    std::conditional_t<ROWS, RowsProduct<T>, Product<T, S == Store::F16 || (F32 && !SUMS), PX, QX, !F32 ? 1 : SUMS ? 6 : 3>> prod;
    if constexpr (ROWS) prod.run(a, rows, p0, q0);
    else prod.run(a.P, Q, p0, q0, k0, k1, smem);

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4, wp = wave % T::WAVES_P, wq = wave / T::WAVES_P;
    const int pw = p0 + wp * T::FP * 16, qw = q0 + wq * T::FQ * 16;     // this wave's corner
    if constexpr (F32 && !ROWS && !SUMS) {         // the rows' powers of two
        int qe[T::FQ];
        bool endless = false;
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) endless |= (qe[j] = a.q_exp[min(qw + 16 * j + n16, rows - 1)]) == kEndless;
#pragma unroll
        for (int i = 0; i < T::FP; ++i) {          // (the array goes on to a tile's end; what stands there changes nothing: the products are 0)
            const i32x4 pe = *(const i32x4*)(a.p_exp + pw + 16 * i + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                endless |= pe[r] == kEndless && pw + 16 * i + 4 * g + r < a.P.size;
#pragma unroll
                for (int j = 0; j < T::FQ; ++j) prod.acc[i][j][r] = __builtin_ldexpf(prod.acc[i][j][r], pe[r] + qe[j]);
            }
        }
        if (__ballot(endless)) whole_logits<T>(prod.acc, a, rows, pw, qw);
    }
    // Exponentials are in base 2, the scale and log2(e) in one factor that is not negative.  Eight waves reach the end of a
    // tile together, so nothing hides these instructions: one maximum, one multiply-add, one exponential (16 cycles) and one addition
    // (or half a conversion) per logit, and everything that only the vocabulary's last tile or a row's target needs is kept out of that.
    float scale2 = a.scale2;
    if (ST != Stage::Dx && ST != Stage::Dw && scale2 < 0.f) {
        scale2 = -scale2;
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int j = 0; j < T::FQ; ++j) prod.acc[i][j] = -prod.acc[i][j];
    }
    const bool whole = p0 + T::BP <= a.P.size;     // no column behind the end of the vocabulary
    // logit y of this wave's columns and row block j, for the lane that has it
    auto pick = [&](int j, int y) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < T::FP; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) x = y == 16 * i + 4 * g + r ? prod.acc[i][j][r] : x;
        return x;
    };
    if constexpr (ST == Stage::Logits) {
        SPH_LDS float* shared = (SPH_LDS float*)smem;                     // [WAVES_P][BQ][2]
        if (!whole) {
#pragma unroll
            for (int i = 0; i < T::FP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (pw + 16 * i + 4 * g + r >= a.P.size)
#pragma unroll
                        for (int j = 0; j < T::FQ; ++j) prod.acc[i][j][r] = -__builtin_inff();
            if (scale2 == 0.f) scale2 = 1e-38f;    // (so that minus infinity stays one)
        }
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) {
            const int q = qw + 16 * j + n16;
            float m = prod.acc[0][j][0];           // (a NaN may get lost here: the sum has it)
#pragma unroll
            for (int i = 0; i < T::FP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = fmaxf(m, prod.acc[i][j][r]);
            m = max_across_groups(m) * scale2;
            const float shift = __builtin_fabsf(m) < __builtin_inff() ? m : 0.f;
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < T::FP; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r & 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(prod.acc[i][j][r], scale2, -shift));
            const float all = sum_across_groups(sum[0] + sum[1]);
            if (g == 0) {
                shared[(wp * T::BQ + q - q0) * 2] = m;
                shared[(wp * T::BQ + q - q0) * 2 + 1] = all;
            }
            if (q < rows) {
                const int y = load_id(a.targets, a.id_bytes, a.rows ? a.rows[q] : q) - pw;
                if (y >= 0 && y < T::FP * 16 && pw + y < a.V && ((y >> 2) & 3) == g) a.target_logit[q] = pick(j, y) * scale2;
            }
        }
        __syncthreads();
        for (int i = tid; i < T::BQ; i += T::THREADS) {
            if (q0 + i >= rows) continue;
            float m = shared[i * 2], sum = 0.f;
            for (int w = 1; w < T::WAVES_P; ++w) m = fmaxf(m, shared[(w * T::BQ + i) * 2]);
            const float shift = __builtin_fabsf(m) < __builtin_inff() ? m : 0.f;
            for (int w = 0; w < T::WAVES_P; ++w) {
                const float mw = shared[(w * T::BQ + i) * 2], s = shared[(w * T::BQ + i) * 2 + 1];
                const float sw = __builtin_fabsf(mw) < __builtin_inff() ? mw : 0.f;   // what s is relative to
                sum += mw == -__builtin_inff() ? s : s * __builtin_amdgcn_exp2f(sw - shift);
            }
            a.partial[(size_t)tile.p * a.partial_ld + q0 + i] = float2{m, sum};
        }
    } else if constexpr (ST == Stage::G) {
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) {
            const int q = qw + 16 * j + n16, qc = min(q, rows - 1);
            const float lse2 = a.g_lse2[qc], gq = a.g[qc];
            const int y = a.g_target[qc] - a.v0 - pw;
            unsigned short* const row = (unsigned short*)a.G + (size_t)qc * a.G_ld + pw;
            auto value = [&](int i, float (&d)[4]) {
#pragma unroll
                for (int r = 0; r < 4; ++r) d[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(prod.acc[i][j][r], scale2, -lse2)) * gq;
                if (__ballot(y >> 4 == i)) {       // a target in these sixteen columns (few have one)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (y == 16 * i + 4 * g + r) d[r] = (__builtin_amdgcn_exp2f(__builtin_fmaf(prod.acc[i][j][r], scale2, -lse2)) - 1.f) * gq;
                }
                if (!whole)
#pragma unroll
                    for (int r = 0; r < 4; ++r) d[r] = pw + 16 * i + 4 * g + r < a.P.size ? d[r] : 0.f;
            };
            // two fragments at a time: lanes exchange halves, so that each has eight neighbouring columns of one and 16 bytes to store
            static_assert(T::FP % 2 == 0, "");
#pragma unroll
            for (int i = 0; i < T::FP; i += 2) {
                float d[2][4];
                value(i, d[0]);
                value(i + 1, d[1]);
                if constexpr (ROWS) {              // fp32 as it is
#pragma unroll
                    for (int f = 0; f < 2; ++f)
                        if (q < rows) *(f32x4*)((float*)a.G + (size_t)qc * a.G_ld + pw + 16 * (i + f) + 4 * g) = f32x4{d[f][0], d[f][1], d[f][2], d[f][3]};
                    continue;
                }
                unsigned short* to = row + 16 * (i + (g & 1)) + 8 * (g >> 1);
                if constexpr (S == Store::F32) {
                    i32x2 part[2][3];              // [fragment][part]
#pragma unroll
                    for (int f = 0; f < 2; ++f) split3(d[f], part[f]);
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        const i32x4 o = join_fragments(part[0][k], part[1][k]);
                        if (q < rows) *(i32x4*)(to + k * a.G_part) = o;
                    }
                } else {
                    const i32x4 o = join_fragments(i32x2{pack2<S == Store::F16>(d[0][0], d[0][1]), pack2<S == Store::F16>(d[0][2], d[0][3])},
                                                   i32x2{pack2<S == Store::F16>(d[1][0], d[1][1]), pack2<S == Store::F16>(d[1][2], d[1][3])});
                    if (q < rows) *(i32x4*)to = o;
                }
            }
        }
    } else {
        // dX: fp32 sums, one array per slice or one that pieces are added to; dW: rows of the result, in its type
        const int limit = ST == Stage::Dx ? rows : a.out_rows;
        const bool pairs = ST == Stage::Dw && S != Store::F32 && (((uintptr_t)a.out | (unsigned)(a.out_ld * 2)) & 15) == 0 && a.out_cols % 8 == 0;
#pragma unroll
        for (int j = 0; j < T::FQ; ++j) {
            const int q = qw + 16 * j + n16;
            if constexpr (ST == Stage::Dw && S != Store::F32) {
                if (pairs) {                       // (as in G)
#pragma unroll
                    for (int i = 0; i < T::FP; i += 2) {
                        const f32x4 x = prod.acc[i][j] * down, z = prod.acc[i + 1][j] * down;
                        const i32x4 o = join_fragments(i32x2{pack2<S == Store::F16>(x[0], x[1]), pack2<S == Store::F16>(x[2], x[3])},
                                                       i32x2{pack2<S == Store::F16>(z[0], z[1]), pack2<S == Store::F16>(z[2], z[3])});
                        const int p = pw + 16 * (i + (g & 1)) + 8 * (g >> 1);
                        if (q < limit && p < a.out_cols) *(i32x4*)((short*)a.out + (size_t)q * a.out_ld + p) = o;
                    }
                    continue;
                }
            }
            if (q >= limit) continue;
#pragma unroll
            for (int i = 0; i < T::FP; ++i) {
                const int p = pw + 16 * i + 4 * g;
                if (p >= a.out_cols) continue;
                if constexpr (ST == Stage::Dx) {   // (out_ld is a multiple of 4)
                    f32x4* to = (f32x4*)((float*)a.out + ((size_t)tile.slice * rows + q) * a.out_ld + p);
                    f32x4 x = prod.acc[i][j];
                    if (a.accumulate) x += *to;
                    *to = x;
                } else {
                    const size_t at = (size_t)q * a.out_ld + p;
                    float x[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = prod.acc[i][j][r] * down;
                    constexpr int N = S == Store::F32 ? 16 : 8;
                    if (p + 4 <= a.out_cols && (((uintptr_t)a.out | (unsigned)(a.out_ld * store_bytes<S>())) & (N - 1)) == 0) {
                        if constexpr (S == Store::F32) *(f32x4*)((float*)a.out + at) = f32x4{x[0], x[1], x[2], x[3]};
                        else *(i32x2*)((short*)a.out + at) = i32x2{pack2<S == Store::F16>(x[0], x[1]), pack2<S == Store::F16>(x[2], x[3])};
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (p + r < a.out_cols) store_el<S>(a.out, at + r, x[r]);
                    }
                }
            }
        }
    }
}

template <class T, Store S, Stage ST>
__global__ __launch_bounds__(T::THREADS, T::FP * T::FQ > 32 ? 1 : 2)
void vocab_tile_kernel(VocabArgs a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    vocab_tile<T, S, ST>(a, blockIdx.x, (SPH_LDS unsigned char*)smem_raw);
}

// dX and dW of a piece, which do not depend on each other, in one launch: dX's tiles first.  For small problems one launch less, and where
// neither fills the chip its round is shared.
template <class T, Store S>
__global__ __launch_bounds__(T::THREADS, T::FP * T::FQ > 32 ? 1 : 2)
void vocab_gradients_kernel(VocabArgs dx, VocabArgs dw, int dx_blocks)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    if ((int)blockIdx.x < dx_blocks) vocab_tile<T, S, Stage::Dx>(dx, blockIdx.x, (SPH_LDS unsigned char*)smem_raw);
    else vocab_tile<T, S, Stage::Dw>(dw, (int)blockIdx.x - dx_blocks, (SPH_LDS unsigned char*)smem_raw);
}

// ---- around the products ---------------------------------------------------------------------------------

// Which rows count (target >= 0), in order: rows[m] = t, place[t] = m or -1; and with `dloss` the scale of their gradients.
enum class Reduce { None, Sum, Mean };             // of dloss: [T], or one value
struct RowArgs {
    const void* targets; int id_bytes; int T;
    int* rows; int* place; VocabInfo* info;
    const float* dloss; Reduce reduce; float scale; int half;   // half: G is stored in fp16
    __device__ __forceinline__ bool by_row() const { return dloss && half && reduce == Reduce::None; }
};

// The power of two that brings |x| to 2^13 .. 2^14
__device__ __forceinline__ float gradient_factor(float x)
{
    x = __builtin_fabsf(x);
    return x > 0.f && x < __builtin_inff() ? __builtin_ldexpf(1.f, max(-126, min(126, 13 - (__builtin_amdgcn_frexp_expf(x) - 1)))) : 1.f;
}

// `top`, `least`: the largest |dloss| of a row that counts and the smallest that is not 0, where there is one for each
__device__ __forceinline__ VocabInfo row_scale(const RowArgs& a, int n, float top, float least)
{
    VocabInfo out{n, 1.f, 1.f, 1};
    if (a.dloss && a.reduce != Reduce::None) {
        // One gradient for all rows comes behind the sums: G is then p - [v = y], and the -1 of a target, which is most of a row's
        // gradient and of a rare id's, has no rounding (with g in front, g (p - 1) is rounded to the type: 2.6e-3 from 64 bits in bf16 where
        // few rows count, 1.7e-3 without).  fp16: 2^14 makes a probability of 2^-28 a normal number still.
        const float g = n ? (a.reduce == Reduce::Mean ? *a.dloss / (float)n : *a.dloss) : 0.f;
        out.up = a.half ? 16384.f : 1.f;
        out.down = g * a.scale / out.up;
    } else if (a.by_row()) {
        // By the largest |c g|.  That keeps dW's sums over the rows to 2^-38 of it; a row of dX has to keep its own gradient's bits, so where the
        // rows' gradients differ dX takes a G of its own, each row brought up by itself.
        out.up = gradient_factor(top * a.scale);
        out.down = 1.f / out.up;
        out.even = top < __builtin_inff() && least >= top * 0.0625f;
    }
    return out;
}

__device__ __forceinline__ float max_over_wave(float x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// |x| among those that `least` is the smallest of
__device__ __forceinline__ float smaller(float least, float x)
{
    x = __builtin_fabsf(x);
    return x > 0.f ? fminf(least, x) : least;
}

__device__ __forceinline__ int lanes_below(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// One workgroup, for more rows than kOwnRows: T ids are little beside what follows.
constexpr int kRowsThreads = 1024;

__global__ __launch_bounds__(kRowsThreads)
void vocab_rows_kernel(RowArgs a)
{
    constexpr int WAVES = kRowsThreads / 64, EACH = 8;      // a wave takes EACH times 64 neighbouring rows at a time
    __shared__ int part[2][WAVES];
    __shared__ float most[WAVES], fewest[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int n = 0, turn = 0;
    float top = 0.f, least = __builtin_inff();
    for (long long t0 = 0; t0 < a.T; t0 += kRowsThreads * EACH, turn ^= 1) {
        const long long t = t0 + wave * (64 * EACH) + lane;
        int id[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) id[i] = t + i * 64 < a.T ? load_id(a.targets, a.id_bytes, t + i * 64) : -1;
        uint64_t counts[EACH];
        int of_wave = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            counts[i] = __ballot(id[i] >= 0);
            of_wave += __builtin_popcountll(counts[i]);
        }
        if (lane == 0) part[turn][wave] = of_wave;
        __syncthreads();
        int at = n;
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) at += part[turn][w];
            n += part[turn][w];
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int m = at + lanes_below(counts[i]);
            if (t + i * 64 < a.T) a.place[t + i * 64] = id[i] >= 0 ? m : -1;
            if (id[i] >= 0) {
                a.rows[m] = (int)(t + i * 64);
                if (a.by_row()) {
                    const float g = a.dloss[t + i * 64];
                    top = fmaxf(top, __builtin_fabsf(g));
                    least = smaller(least, g);
                }
            }
            at += __builtin_popcountll(counts[i]);
        }
    }
    top = max_over_wave(top);
    least = -max_over_wave(-least);
    if (lane == 0) most[wave] = top, fewest[wave] = least;
    __syncthreads();
    if (tid != 0) return;
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, most[w]), least = fminf(least, fewest[w]);
    *a.info = row_scale(a, n, top, least);
}

// Rows as the products want them: 16-bit, 16-byte aligned, whole pieces of 8; gathered if only some count; fp32 in two
// parts.  One wave per row; X's and W's in one launch.  For at most kOwnRows rows each workgroup finds out by itself which rows before its
// own count, which spares a launch of one workgroup in front.
constexpr int kPackThreads = 256, kPackRows = kPackThreads / 64, kOwnRows = 1024;

struct PackRows {
    const void* in; void* out; int n, D, ld;       // (ld: elements per row of out, a multiple of 8)
    long long part;                                // elements from part to part
    void* sum_out;                                 // fp32: the three parts that the products with G take, or NULL
    int* exp;                                      // fp32: for the logits, the power of two that the row was divided by
};
struct PackArgs {
    PackRows x, w;
    int x_groups;                                  // workgroups on X, the rest on W
    int compact, own_rows;                         // only X's rows that count; found here
    RowArgs r;
    const float* lse; int* g_target; float* g_lse2; float* g;   // what the G stage needs of each row, or NULL
    float *g_own, *own_down;                       // fp16, one gradient per row: g of dX's own G and the factor of dX's rows, or NULL
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

template <Store S>
__global__ __launch_bounds__(kPackThreads)
void vocab_pack_kernel(PackArgs a)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool on_x = (int)blockIdx.x < a.x_groups;
    if (!on_x) {
        const long long v = (long long)((int)blockIdx.x - a.x_groups) * kPackRows + wave;
        if (v < a.w.n) pack_row<S>(a.w, v, v, lane);
        return;
    }
    const long long row = (long long)blockIdx.x * kPackRows + wave;
    long long t = row, m = row;
    float up = 1.f;
    int even = 1;
    if (a.compact && a.own_rows) {
        __shared__ int before[kPackRows], all[kPackRows];
        __shared__ float most[kPackRows], fewest[kPackRows];
        const int t0 = (int)blockIdx.x * kPackRows;
        int b = 0, n = 0;
        float top = 0.f, least = __builtin_inff();
        for (int i0 = 0; i0 < a.r.T; i0 += kPackThreads) {
            const int i = i0 + tid;
            const bool counts = i < a.r.T && load_id(a.r.targets, a.r.id_bytes, i) >= 0;
            n += __builtin_popcountll(__ballot(counts));
            b += __builtin_popcountll(__ballot(counts && i < t0));
            if (counts && a.r.by_row()) {
                const float g = a.r.dloss[i];
                top = fmaxf(top, __builtin_fabsf(g));
                least = smaller(least, g);
            }
        }
        if (a.r.by_row()) {
            top = max_over_wave(top);
            least = -max_over_wave(-least);
        }
        if (lane == 0) before[wave] = b, all[wave] = n, most[wave] = top, fewest[wave] = least;
        __syncthreads();
        b = n = 0;
        for (int w = 0; w < kPackRows; ++w) b += before[w], n += all[w], top = fmaxf(top, most[w]), least = fminf(least, fewest[w]);
        const VocabInfo info = row_scale(a.r, n, top, least);
        if (blockIdx.x == 0 && tid == 0) *a.r.info = info;
        if (row >= a.r.T) return;
        const bool counts = load_id(a.r.targets, a.r.id_bytes, row) >= 0;
        m = b;
        for (int i = t0; i < row; ++i) m += load_id(a.r.targets, a.r.id_bytes, i) >= 0;
        if (lane == 0) a.r.place[row] = counts ? (int)m : -1;
        if (!counts) return;
        if (lane == 0) a.r.rows[m] = (int)row;
        up = info.up;
        even = info.even;
    } else if (a.compact) {
        if (m >= a.r.info->rows) return;
        t = a.r.rows[m];
        up = a.r.info->up;
        even = a.r.info->even;
    } else if (m >= a.x.n) {
        return;
    }
    if (a.g_target && lane == 0) {
        a.g_target[m] = load_id(a.r.targets, a.r.id_bytes, t);
        a.g_lse2[m] = a.lse[t] * kLog2e;
        const float g = a.r.reduce == Reduce::None ? a.r.dloss[t] * a.r.scale : 1.f;
        a.g[m] = g * up;
        if (a.g_own) {
            const float own = even ? up : gradient_factor(g);
            a.g_own[m] = g * own;
            a.own_down[m] = 1.f / own;
        }
    }
    pack_row<S>(a.x, t, m, lane);
}

// The tiles' maxima and sums joined: 2^log_rows rows per workgroup (64 at most), its other lanes and waves a share of the tiles each.
// One row in a workgroup of one lane per row and wave took 7.8 us for 256 tiles, each wave 32 of them one after another; spread over the lanes
// it is the latency of a load and nine exchanges.  One workgroup on all rows also gives their sum or mean.
constexpr int kJoinLossThreads = 512;

struct LogSum { float top, sum; };                 // sum of exponentials relative to a finite top, or to 0 where it is not finite
__device__ __forceinline__ LogSum join_sums(LogSum a, LogSum b)
{
    auto finite = [](float x) { return __builtin_fabsf(x) < __builtin_inff() ? x : 0.f; };
    const float now = fmaxf(a.top, b.top), c = finite(now);
    auto part = [&](LogSum x) { return x.top == -__builtin_inff() ? x.sum : x.sum * __builtin_amdgcn_exp2f(finite(x.top) - c); };
    return LogSum{now, part(a) + part(b)};
}

__global__ __launch_bounds__(kJoinLossThreads)
void vocab_join_kernel(const float2* __restrict__ partial, int partial_ld, int tiles, int log_rows, const float* __restrict__ target_logit,
                       const void* __restrict__ targets, int id_bytes, const int* __restrict__ place,
                       int all_rows, float* __restrict__ losses, float* __restrict__ lse, float* __restrict__ mean, int divide, int T, int V)
{
    constexpr int W = kJoinLossThreads / 64;
    __shared__ LogSum shared[W][64];
    const int tid = threadIdx.x, wave = tid >> 6, R = 1 << log_rows, row = tid & (R - 1);
    const long long t = ((long long)blockIdx.x << log_rows) + row;
    const int m = t >= T ? -1 : place ? place[t] : (int)t;
    LogSum s{-__builtin_inff(), 0.f};
    if (m >= 0) {
#pragma unroll 4
        for (int i = tid >> log_rows; i < tiles; i += kJoinLossThreads >> log_rows) {
            const float2 x = partial[(size_t)i * partial_ld + m];
            s = join_sums(s, LogSum{x.x, x.y});
        }
    }
    for (int d = R; d < 64; d <<= 1) s = join_sums(s, LogSum{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)});
    if ((tid & 63) < R) shared[wave][row] = s;
    __syncthreads();
    if (wave != 0) return;
    const int y = tid < R && t < T ? load_id(targets, id_bytes, t) : -1;
    float of_row = 0.f;
    if (tid < R && t < T) {
        float l = 0.f;
        if (m >= 0 && (all_rows || y >= 0)) {
            for (int w = 1; w < W; ++w) s = join_sums(s, shared[w][row]);
            const float l2 = (__builtin_fabsf(s.top) < __builtin_inff() ? s.top : 0.f) + __builtin_amdgcn_logf(s.sum);
            l = y >= V ? __builtin_nanf("") : l2 * kLn2;
            if (y >= 0) of_row = y >= V ? __builtin_nanf("") : (l2 - target_logit[m]) * kLn2;
        }
        if (lse) lse[t] = l;
        losses[t] = of_row;
    }
    if (!mean) return;                             // (with one workgroup only)
    double sum = of_row;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    const int n = __builtin_popcountll(__ballot(y >= 0));
    if (tid == 0) *mean = (float)(!divide ? sum : n > 0 ? sum / n : 0.0);
}

// Their sum over the rows that count and its mean: one workgroup, in fp64.  No row that counts: 0.
__global__ __launch_bounds__(1024)
void vocab_mean_kernel(const float* __restrict__ losses, const void* __restrict__ targets, int id_bytes, int T, float* __restrict__ mean, int divide)
{
    __shared__ double shared[2][16];
    const int tid = threadIdx.x;
    double sum = 0.0, n = 0.0;
    for (long long t = tid; t < T; t += 1024) {
        sum += losses[t];
        n += load_id(targets, id_bytes, t) >= 0;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        sum += __shfl_xor(sum, d);
        n += __shfl_xor(n, d);
    }
    if ((tid & 63) == 0) {
        shared[0][tid >> 6] = sum;
        shared[1][tid >> 6] = n;
    }
    __syncthreads();
    if (tid != 0) return;
    for (int w = 1; w < 16; ++w) {
        sum += shared[0][w];
        n += shared[1][w];
    }
    *mean = (float)(!divide ? sum : n > 0.0 ? sum / n : 0.0);
}

// dX: the slices' sums, in order, scaled back and rounded; zeros for rows that do not count.  One wave per row and 256 columns, eight slices'
// loads under way.  (64 slices of 17 x 1024, one after the other: 113 us.)
constexpr int kDxCols = 256;

template <Store S>
__global__ __launch_bounds__(256)
void vocab_dx_kernel(const float* __restrict__ part, int slices, int ld, int tile_q, int tiles_p, int target, const int* __restrict__ place,
                     const VocabInfo* __restrict__ info, const float* __restrict__ own_down, void* __restrict__ dX, int T, int D)
{
    const int lane = threadIdx.x & 63;
    const long long t = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= T) return;
    const int m = place[t];
    const int rows = info->rows;
    const size_t slice = (size_t)rows * ld;
    slices = dx_slices(rows, T, slices, tile_q, tiles_p, target);
    const bool wide = ((uintptr_t)dX & 15) == 0 && D % 4 == 0;
    const int c = (int)blockIdx.y * kDxCols + lane * 4;
    if (c < D) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (m >= 0) {
            const float* from = part + (size_t)m * ld + c;
            constexpr int AHEAD = 8;
            for (int s0 = 0; s0 < slices; s0 += AHEAD) {
                f32x4 y[AHEAD];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) y[a] = *(const f32x4*)(from + min(s0 + a, slices - 1) * slice);
#pragma unroll
                for (int a = 0; a < AHEAD; ++a)
                    if (s0 + a < slices) x += y[a];
            }
            x *= own_down ? own_down[m] : info->down;   // (not of rows that do not count: it may be infinite or NaN, and their gradient is 0)
        }
        const size_t at = (size_t)t * D + c;
        if (wide) {
            if constexpr (S == Store::F32) *(f32x4*)((float*)dX + at) = x;
            else *(i32x2*)((short*)dX + at) = i32x2{pack2<S == Store::F16>(x[0], x[1]), pack2<S == Store::F16>(x[2], x[3])};
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (c + r < D) store_el<S>(dX, at + r, x[r]);
        }
    }
}

}  // namespace sphattn
