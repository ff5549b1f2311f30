// Embedding lookup with scaling and the gradient of the table by sorted tokens, for gfx950.
//
//   O[t] = s m_t E[x_t]          dE[v] = s sum_{t : x_t = v} m_t dO[t]
//
// Both are bound by memory: the lookup reads and writes T D values, the gradient reads T D and writes
// V D.  What the gradient needs beside that is an order in which equal tokens are neighbours, without atomics
// on floats (their order, and with it the result, would change from run to run).
#pragma once
#include "sphattn_store.hpp"

namespace sphattn {

// ---- lookup ------------------------------------------------------------------------------------------
// One wave per row, four rows per workgroup; a lane moves 16 bytes at a time, four of them under way.  WIDE: rows
// are whole 16-byte pieces from an aligned start on.  Bound by memory (16384 rows of 2048 bf16 20 us, 6.5 TB/s with common rows from the
// caches), and for few rows by the launch (one row: kernel 1.6 us).
constexpr int kEmbedThreads = 256;

template <Store S, bool WIDE>
__global__ __launch_bounds__(kEmbedThreads)
void embed_fwd_kernel(const void* __restrict__ tokens, int id_bytes, const void* __restrict__ table,
                      const float* __restrict__ mult, void* __restrict__ O, int T, int V, int D, float scale)
{
    const int lane = threadIdx.x & 63;
    constexpr int WAVES = kEmbedThreads / 64;
    for (long long row = (long long)blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); row < T; row += (long long)gridDim.x * WAVES) {
        const int v = load_id(tokens, id_bytes, row);
        // no token: zeros; not a token of this table: NaN.  Both without reading the table.
        const bool in = v >= 0 && v < V;
        const float f = in ? (mult ? mult[row] * scale : scale) : 0.f;
        const float fill = v < 0 ? 0.f : __builtin_nanf("");
        constexpr int N = per16<S>(), AHEAD = 4;
        const size_t src = (size_t)(in ? v : 0) * D, dst = (size_t)row * D;
        for (int c0 = lane * N; c0 < D; c0 += 64 * N * AHEAD) {
            i32x4 w[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int c = c0 + a * 64 * N;
                w[a] = i32x4{0, 0, 0, 0};
                if (in && c < D) w[a] = load16<S, WIDE>(table, src + c, D - c, (size_t)V * D - src - c);
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int c = c0 + a * 64 * N;
                float x[N];
                widen16<S>(w[a], x);
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = in ? x[i] * f : fill;
                if (c < D) store16<S, WIDE>(O, dst + c, narrow16<S>(x), D - c);
            }
        }
    }
}

// ---- gradient: sorting ---------------------------------------------------------------------------------
// A stable counting sort of the positions by token in one launch: a workgroup owns `ids` neighbouring
// token ids and reads all T tokens twice (they stay in the caches: 64 bytes a cycle and CU, 0.25 us per 4096
// of 8 bytes).  First it counts, per wave (each wave has a stretch of t of its own) and id, its own ids, and how many
// tokens lie below them, which is where its part of the result begins; the second time each position goes to its place:
// that of its id and wave, plus its rank among the equal tokens before it in the wave.  No workgroup waits for
// another, no atomic touches memory.  8192 tokens of 19999 ids 14 us, 8 of them the zeros; 32768 of 5003 20 us, bound by the instructions per
// token.  Then it writes zeros to those rows of the gradient that have no token.
//   first : [V + 1], where the positions of id v begin in `sorted`;  sorted : [T]
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortMaxIds = 512;

constexpr int sort_lds_bytes(int ids) { return (kSortWaves * ids + 2 * kSortWaves + 2) * 4; }

// sum of x over the lanes below, and `total` over all
__device__ __forceinline__ int exclusive_over_wave(int x, int lane, int& total)
{
    int s = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(s, d);
        if (lane >= d) s += y;
    }
    total = __shfl(s, 63);
    return s - x;
}

__global__ __launch_bounds__(kSortThreads)
void embed_sort_kernel(const void* __restrict__ tokens, int id_bytes, int* __restrict__ first, int* __restrict__ sorted,
                       void* __restrict__ dtable, int T, int V, int ids, int row_bytes)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    int* cnt = (int*)smem_raw;                     // [kSortWaves][ids]
    int* part = cnt + kSortWaves * ids;            // [2][kSortWaves]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lo = blockIdx.x * ids, n_ids = min(ids, V - lo);
    for (int i = tid; i < kSortWaves * ids; i += kSortThreads) cnt[i] = 0;
    __syncthreads();

    // this wave's tokens: whole batches of 64
    const long long batches = ((long long)T + 63) / 64, share = (batches + kSortWaves - 1) / kSortWaves;
    const long long t0 = min((long long)T, wave * share * 64), t1 = min((long long)T, t0 + share * 64);
    int* mine = cnt + wave * ids;
    // Eight times 64 positions at a time; one round per different own id among them, over all eight.  (One LDS access per id and eight batches
    // instead of one per batch: each waits for the one before it, and a token at half of 32768 positions made 32 us of them.)
    constexpr int AHEAD = 8;
    int below = 0, next[AHEAD];
    // One turn before they are needed.  Every workgroup does this with every token, so instructions count: 64 tokens took 45 of them with a
    // check and 64-bit comparisons at each load (32768 tokens 30 us).  What is no id of the table becomes -1.
    auto fetch = [&](long long t) {
        if (t + 64 * AHEAD > t1) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) next[a] = t + a * 64 + lane < t1 ? load_id(tokens, id_bytes, t + a * 64 + lane) : -1;
        } else if (id_bytes == 4) {
            const int* from = (const int*)tokens + t + lane;
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) next[a] = from[a * 64];
        } else {
            const int2* from = (const int2*)tokens + t + lane;
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int2 x = from[a * 64];
                next[a] = x.y == 0 ? x.x : -1;
            }
        }
    };
    auto each_id = [&](const int (&v)[AHEAD], auto&& round) {
        uint64_t left[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) left[a] = __ballot((unsigned)(v[a] - lo) < (unsigned)n_ids);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            while (left[a]) {
                const int id = __builtin_amdgcn_readlane(v[a], __builtin_ctzll(left[a]));
                uint64_t same[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    same[k] = k < a ? 0 : __ballot(v[k] == id);
                    left[k] &= ~same[k];
                }
                round(id, same);
            }
        }
    };
    fetch(t0);
    for (long long t = t0; t < t1; t += 64 * AHEAD) {
        int v[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) v[a] = next[a];
        fetch(t + 64 * AHEAD);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) below += __builtin_popcountll(__ballot((unsigned)v[a] < (unsigned)lo));
        each_id(v, [&](int id, const uint64_t (&same)[AHEAD]) {
            int n = 0;
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) n += __builtin_popcountll(same[a]);
            if (lane == 0) mine[id - lo] += n;     // (no other wave has this row of counts)
        });
    }
    if (lane == 0) part[wave] = below;
    __syncthreads();

    // places: ids in order, within an id the waves in order.  Thread i has id i (ids <= kSortThreads).
    int of_id = 0;
    if (tid < n_ids)
        for (int w = 0; w < kSortWaves; ++w) of_id += cnt[w * ids + tid];
    int of_wave, base = 0;
    int at = exclusive_over_wave(of_id, lane, of_wave);
    if (lane == 0) part[kSortWaves + wave] = of_wave;
    __syncthreads();
    for (int w = 0; w < kSortWaves; ++w) {
        base += part[w];
        if (w < wave) at += part[kSortWaves + w];
    }
    at += base;
    if (tid < n_ids) {
        first[lo + tid] = at;
        if (lo + tid == V - 1) first[V] = at + of_id;
        int p = at;
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = cnt[w * ids + tid];
            cnt[w * ids + tid] = p;
            p += c;
        }
    }
    __syncthreads();

    fetch(t0);
    for (long long t = t0; t < t1; t += 64 * AHEAD) {
        int v[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) v[a] = next[a];
        fetch(t + 64 * AHEAD);
        each_id(v, [&](int id, const uint64_t (&same)[AHEAD]) {
            int p = mine[id - lo];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                if (v[a] == id) sorted[p + __builtin_amdgcn_mbcnt_hi((uint32_t)(same[a] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same[a], 0))] = (int)(t + a * 64 + lane);
                p += __builtin_popcountll(same[a]);
            }
            mine[id - lo] = p;                     // (every lane the same value)
        });
    }

    // rows without a token, a wave each; thread i says over LDS how many id i has
    __syncthreads();
    if (tid < n_ids) cnt[tid] = of_id;
    __syncthreads();
    for (int i = wave; i < n_ids; i += kSortWaves) {
        if (cnt[i] != 0) continue;
        unsigned char* row = (unsigned char*)dtable + (size_t)(lo + i) * row_bytes;
        if ((((uintptr_t)dtable | (unsigned)row_bytes) & 15) == 0) {
            for (int c = lane; c < row_bytes / 16; c += 64) ((i32x4*)row)[c] = i32x4{0, 0, 0, 0};
        } else {
            for (int c = lane; c < row_bytes / 2; c += 64) ((short*)row)[c] = 0;
        }
    }
}

// ---- gradient: sums ------------------------------------------------------------------------------------
// The sorted positions are cut into pieces of `len`, whatever tokens they hold, so a token that half of all positions have is
// shared by as many waves as it fills pieces.  A wave adds up a piece's runs of equal tokens over 64 lanes' columns in fp32.  A
// run that lies inside the piece is a row of the gradient; one that crosses its borders leaves a partial sum: [piece][0] if
// it began before the piece, [piece][1] if it begins in it and goes on behind it.  Bound by memory where rows are many (32768 x 512 fp32 14 us,
// 4.7 TB/s), by the chain position, token, row where they are few (8192 x 1024 bf16 9 us, 1.9 TB/s).
__host__ __device__ constexpr int partial_ld(int D) { return (D + 7) / 8 * 8; }   // floats per row of partial sums

template <Store S, bool WIDE>
__global__ __launch_bounds__(kEmbedThreads)
void embed_sum_kernel(const void* __restrict__ tokens, int id_bytes, const float* __restrict__ mult, const void* __restrict__ dO,
                      const int* __restrict__ first, const int* __restrict__ sorted, float* __restrict__ partial,
                      void* __restrict__ dtable, int T, int V, int D, float scale, int len, int n_pieces)
{
    constexpr int C = per16<S>(), AHEAD = 8;
    const int lane = threadIdx.x & 63;
    const long long piece = (long long)blockIdx.x * (kEmbedThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (piece >= n_pieces) return;
    const int total = first[V];
    const long long p0 = piece * len, p1 = min((long long)total, p0 + len);
    if (p0 >= p1) return;
    const int col = ((int)blockIdx.y * 64 + lane) * C;
    const bool live = col < D;
    float acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i) acc[i] = 0.f;
    int run = -1, r0 = 0, r1 = 0;                  // the id that acc belongs to, and where its positions begin and end
    auto flush = [&](int id) {
        if (live) {
            if (r0 >= p0 && r1 <= p1) store16<S, WIDE>(dtable, (size_t)id * D + col, narrow16<S>(acc), D - col);
            else {
                float* to = partial + ((size_t)piece * 2 + (r0 < p0 ? 0 : 1)) * partial_ld(D) + col;
#pragma unroll
                for (int i = 0; i < C; ++i) to[i] = acc[i];
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) acc[i] = 0.f;
    };
    for (long long b = p0; b < p1; b += 64) {
        // 64 positions, their tokens and factors, one per lane
        const int n = (int)min((long long)64, p1 - b);
        int t = 0, id = 0, begin = 0, end = 0;
        float f = 0.f;
        if (lane < n) {
            t = sorted[b + lane];
            id = load_id(tokens, id_bytes, t);
            f = mult ? mult[t] * scale : scale;
            begin = first[id];                     // (here for all at once: at a run's end each would be waited for)
            end = first[id + 1];
        }
        for (int j0 = 0; j0 < n; j0 += AHEAD) {
            i32x4 w[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const size_t at = (size_t)__builtin_amdgcn_readlane(t, min(j0 + a, n - 1)) * D + col;
                w[a] = i32x4{0, 0, 0, 0};
                if (live) w[a] = load16<S, WIDE>(dO, at, D - col, (size_t)T * D - at);
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                if (j0 + a >= n) break;
                const int v = __builtin_amdgcn_readlane(id, j0 + a);
                const float fa = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), j0 + a));
                if (v != run) {
                    if (run >= 0) flush(run);
                    run = v;
                    r0 = __builtin_amdgcn_readlane(begin, j0 + a);
                    r1 = __builtin_amdgcn_readlane(end, j0 + a);
                }
                float x[C];
                widen16<S>(w[a], x);
#pragma unroll
                for (int i = 0; i < C; ++i) acc[i] = __builtin_fmaf(x[i], fa, acc[i]);
            }
        }
    }
    flush(run);
}

// A row whose run crosses borders: the piece in which it begins adds its partial sums up, eight waves a share of the
// pieces each, sixteen (eight) pieces' loads under way, the shares in order behind that.  512 partial sums of 512 columns 12 us:
// two CUs read them all.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;

template <Store S, bool WIDE>
__global__ __launch_bounds__(kJoinThreads)
void embed_join_kernel(const void* __restrict__ tokens, int id_bytes, const int* __restrict__ first, const int* __restrict__ sorted,
                       const float* __restrict__ partial, void* __restrict__ dtable, int V, int D, int len)
{
    constexpr int C = per16<S>();
    __shared__ float shared[kJoinWaves][64 * C];
    const long long piece = blockIdx.x, p0 = piece * len, p1 = p0 + len;
    if (p1 >= first[V]) return;                    // nothing behind this piece
    const int id = load_id(tokens, id_bytes, sorted[p1 - 1]);
    const int r0 = first[id], r1 = first[id + 1];
    if (r0 < p0 || r1 <= p1) return;               // its last run began earlier, or ends with it
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = ((int)blockIdx.y * 64 + lane) * C;
    const long long last = (r1 - 1) / len;         // the run's last piece
    float acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i) acc[i] = 0.f;
    const long long n = last - piece + 1, share = (n + kJoinWaves - 1) / kJoinWaves;
    const long long q0 = piece + wave * share, q1 = min(last + 1, q0 + share);
    if (col < D) {
        constexpr int AHEAD = S == Store::F32 ? 16 : 8;
        for (long long q = q0; q < q1; q += AHEAD) {
            float x[AHEAD][C];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const long long at = min(q + a, q1 - 1);   // (loads without a condition: none waits for another)
                const float* from = partial + ((size_t)at * 2 + (at == piece ? 1 : 0)) * partial_ld(D) + col;
#pragma unroll
                for (int i = 0; i < C; ++i) x[a][i] = from[i];
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a)
#pragma unroll
                for (int i = 0; i < C; ++i) acc[i] += q + a < q1 ? x[a][i] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) shared[wave][lane * C + i] = acc[i];
    __syncthreads();
    if (wave == 0 && col < D) {
        for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
            for (int i = 0; i < C; ++i) acc[i] += shared[w][lane * C + i];
        store16<S, WIDE>(dtable, (size_t)id * D + col, narrow16<S>(acc), D - col);
    }
}

}  // namespace sphattn
