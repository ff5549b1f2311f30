// Host side of the C ABI declared in include/sphattn_train.h: argument checks, choice of tiles, launches on the
// caller's stream.  Allocates nothing and never synchronises.
#include "sphattn_embed.hpp"
#include "sphattn_vocab.hpp"
#include "sphattn_clip.hpp"
#include "../../include/sphattn_train.h"

#include <climits>
#include <cmath>
#include <stdint.h>

#include <atomic>

namespace {

using namespace sphattn;

constexpr int kCus = 256;

// A range of bytes that a call reads or writes.
struct Range { const void* at; size_t bytes; };

bool meet(const Range& a, const Range& b)
{
    if (!a.at || !b.at || !a.bytes || !b.bytes) return false;
    const uintptr_t a0 = (uintptr_t)a.at, b0 = (uintptr_t)b.at;
    return a0 <= b0 ? b0 - a0 < a.bytes : a0 - b0 < b.bytes;
}

// Each written range against everything else.
template <int W, int R>
bool any_meet(const Range (&written)[W], const Range (&read)[R])
{
    for (int i = 0; i < W; ++i) {
        for (int j = i + 1; j < W; ++j)
            if (meet(written[i], written[j])) return true;
        for (int j = 0; j < R; ++j)
            if (meet(written[i], read[j])) return true;
    }
    return false;
}

bool off(const void* p, size_t alignment) { return ((uintptr_t)p & (alignment - 1)) != 0; }

int element_bytes(int dtype)
{
    return dtype == SPHATTN_F32 ? 4 : dtype == SPHATTN_BF16 || dtype == SPHATTN_F16 ? 2 : 0;
}

int launched() { return hipGetLastError() == hipSuccess ? SPHATTN_OK : SPHATTN_ERR_LAUNCH; }

// A kernel with more than 64 KB of LDS needs its limit raised once per device.  `done` is the kernel's own: kernels of one type
// share whatever a template over the type keeps.
template <typename Kern>
bool raise_lds_limit(Kern kern, int lds_bytes, std::atomic<uint64_t>& done)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
        (void)hipGetLastError();
        return false;
    }
    const uint64_t bit = 1ull << dev;
    if (done.load(std::memory_order_acquire) & bit) return true;
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    done.fetch_or(bit, std::memory_order_release);
    return true;
}

// Pieces of a workspace, each on a 256-byte line.
class Carve {
public:
    explicit Carve(void* base) : base_((unsigned char*)base) {}
    template <typename T> T* take(size_t count)
    {
        T* p = base_ ? (T*)(base_ + used_) : nullptr;
        used_ += (count * sizeof(T) + 255) / 256 * 256;
        return p;
    }
    size_t used() const { return used_; }
private:
    unsigned char* base_;
    size_t used_ = 0;
};

// ---- embedding -------------------------------------------------------------------------------------

bool embed_shape(int T, int V, int D) { return T >= 0 && V >= 1 && V <= 1 << 30 && D >= 1 && D <= 65536; }

int embed_check(const void* tokens, int id_bytes, const float* mult, int T, int V, int D, int dtype)
{
    if (!embed_shape(T, V, D)) return SPHATTN_ERR_SHAPE;
    if (!element_bytes(dtype) || (id_bytes != 4 && id_bytes != 8)) return SPHATTN_ERR_DTYPE;
    if (T > 0 && !tokens) return SPHATTN_ERR_NULL;
    if (off(tokens, id_bytes) || off(mult, 4)) return SPHATTN_ERR_ALIGN;
    return SPHATTN_OK;
}

struct EmbedPlan {
    int ids, sort_groups;                          // token ids per sorting workgroup, workgroups
    int len, pieces;                               // sorted positions per piece, pieces
    int* first;
    int* sorted;
    float* partial;
    size_t bytes;
};

EmbedPlan embed_plan(int T, int V, int D, void* workspace)
{
    EmbedPlan p;
    // one sorting workgroup per CU if ids allow it: each reads all tokens whatever its share
    p.ids = (V + kCus - 1) / kCus;
    p.ids = p.ids < kSortMaxIds ? p.ids : kSortMaxIds;
    p.sort_groups = (V + p.ids - 1) / p.ids;
    // pieces of 16 positions: a wave has 16 rows to add up, eight of them under way.  Longer ones once four waves per CU have work (of 512
    // columns of two bytes each): that many reach memory's rate, and a run over many pieces has fewer partial sums to join.
    p.len = 16;
    while (((long long)T + p.len - 1) / p.len * ((D + 511) / 512) > 4 * kCus && p.len < 1 << 20) p.len *= 2;
    p.pieces = (int)(((long long)T + p.len - 1) / p.len);
    Carve c(workspace);
    p.first = c.take<int>((size_t)V + 1);
    p.sorted = c.take<int>(T);
    p.partial = c.take<float>((size_t)p.pieces * 2 * partial_ld(D));
    p.bytes = c.used();
    return p;
}

template <Store S>
int run_embed_fwd(const void* tokens, int id_bytes, const void* table, const float* mult, void* O, int T, int V, int D, float scale, hipStream_t stream)
{
    const bool wide = !off(table, 16) && !off(O, 16) && D % per16<S>() == 0;
    const long long groups = ((long long)T + 3) / 4, most = 1 << 22;   // (a launch has less than 2^32 threads)
    const dim3 grid((unsigned)(groups < most ? groups : most));
    if (wide) hipLaunchKernelGGL((embed_fwd_kernel<S, true>), grid, dim3(kEmbedThreads), 0, stream, tokens, id_bytes, table, mult, O, T, V, D, scale);
    else hipLaunchKernelGGL((embed_fwd_kernel<S, false>), grid, dim3(kEmbedThreads), 0, stream, tokens, id_bytes, table, mult, O, T, V, D, scale);
    return launched();
}

template <Store S, bool WIDE>
int run_embed_sums(const EmbedPlan& p, const void* tokens, int id_bytes, const float* mult, const void* dO, void* dtable, int T, int V, int D, float scale, hipStream_t stream)
{
    const unsigned columns = (unsigned)((D + 64 * per16<S>() - 1) / (64 * per16<S>()));
    hipLaunchKernelGGL((embed_sum_kernel<S, WIDE>), dim3((unsigned)(p.pieces + 3) / 4, columns), dim3(kEmbedThreads), 0, stream,
                       tokens, id_bytes, mult, dO, p.first, p.sorted, p.partial, dtable, T, V, D, scale, p.len, p.pieces);
    if (p.pieces > 1)
        hipLaunchKernelGGL((embed_join_kernel<S, WIDE>), dim3((unsigned)p.pieces - 1, columns), dim3(kJoinThreads), 0, stream,
                           tokens, id_bytes, p.first, p.sorted, p.partial, dtable, V, D, p.len);
    return launched();
}

template <Store S>
int run_embed_bwd(const EmbedPlan& p, const void* tokens, int id_bytes, const float* mult, const void* dO, void* dtable, int T, int V, int D, float scale, hipStream_t stream)
{
    hipLaunchKernelGGL(embed_sort_kernel, dim3((unsigned)p.sort_groups), dim3(kSortThreads), (size_t)sort_lds_bytes(p.ids), stream,
                       tokens, id_bytes, p.first, p.sorted, dtable, T, V, p.ids, D * store_bytes<S>());
    const int rc = launched();
    if (rc != SPHATTN_OK || T == 0) return rc;
    const bool wide = !off(dO, 16) && !off(dtable, 16) && D % per16<S>() == 0;
    return wide ? run_embed_sums<S, true>(p, tokens, id_bytes, mult, dO, dtable, T, V, D, scale, stream)
                : run_embed_sums<S, false>(p, tokens, id_bytes, mult, dO, dtable, T, V, D, scale, stream);
}

// ---- vocabulary loss ---------------------------------------------------------------------------------

using Big = Tile<256, 256, 2, 4, 4>;               // eight waves of 128 x 64: one workgroup per CU
using Mid = Tile<128, 128, 2, 2, 4>;               // four of 64 x 64: two per CU
using Low = Tile<128, 64, 4, 1, 4>;                // up to 64 rows
using Few = Tile<128, 32, 4, 1, 4>;                // fp32: up to 32 rows (17 x 50000 x 1024 logits 111 -> 68 us: its matrix instruction is the slow one)
using One = Tile<128, 16, 4, 1, 6>;                // up to 16 rows

// Of G (or, where that is more, of X): what the last-level cache holds, and half as much again where one piece is enough then.  (One piece instead of
// two: 8000 rows, 20011 ids, 320 MB 1387 -> 1354 us, with 1200 rows that count 313 -> 287; 8192 x 23000, 377 MB 878 -> 820; but 8192 x 32768, 537 MB
// 1978 -> 2018, and 65536 ids in three pieces instead of four 7170 -> 7330.)
constexpr size_t kPieceBytes = 256u << 20, kOnePieceBytes = 400u << 20;

bool vocab_shape(int T, int V, int D) { return T >= 0 && T <= 1 << 20 && V >= 1 && V <= 1 << 24 && D >= 1 && D <= 65536; }

long long up_to(long long x, long long m) { return (x + m - 1) / m * m; }

// The tile of fewest rounds of the CUs' time: a Mid tile takes 0.36 of a Big one's in a CU that runs two of them
bool big_tiles(long long p, long long q)
{
    const long long big = ((p + 255) / 256) * ((q + 255) / 256), mid = ((p + 127) / 128) * ((q + 127) / 128);
    const double big_time = (double)((big + kCus - 1) / kCus), mid_time = 0.72 * (double)((mid + 2 * kCus - 1) / (2 * kCus));
    return big_time <= mid_time;
}

struct Vocab {
    int T, V, D, parts, ld;                        // parts: of X and W for the logits; ld: elements per packed row
    int piece, n_pieces, g_parts;                  // backward: vocabulary ids of a piece of G, its 16-bit parts
    bool dx_big; int slices;                       // dX: its tile, slices of its sum over a piece
    // workspace
    VocabInfo* info;
    int *x_exp, *w_exp;                            // fp32 in parts
    int *rows, *place, *g_target;
    float *g_lse2, *g, *target_logit, *dx;
    float *g_own, *own_down;                       // fp16
    float2* partial;
    unsigned short *x, *w, *G;
    unsigned short *x_sum, *w_sum;                 // fp32 with parts: what G is multiplied with
    size_t bytes;
};

// dX's tile and the slices of its sum over n ids, by the time that its rounds take: in a round of 256 Big tiles each takes 27 ns per id,
// in one of 512 Mid tiles 20, and every slice is written and read again as fp32.  (8192 rows, width 1024: 512 Mid tiles 338 us per 16384 ids,
// 256 Big ones in two slices 225.)
void dx_choice(long long T, long long ld, int n, bool& big, int& slices)
{
    double best = 0.0;
    for (int b = 1; b >= 0; --b) {
        const int tile = b ? 256 : 128, at_once = b ? kCus : 2 * kCus;
        const long long tiles = ((T + tile - 1) / tile) * ((ld + tile - 1) / tile);
        for (int s = 1; s <= 64 && (s == 1 || n / s >= 512); s *= 2) {
            const double rounds = (double)((tiles * s + at_once - 1) / at_once);
            const double us = rounds * (n / s) * (b ? 0.027 : 0.020) + s * (double)(T * ld) * 8.0 / 4.5e6;
            if (best == 0.0 || us < best) best = us, big = b, slices = s;
        }
    }
}

// fp32 and few rows: kernels that read fp32 as it is
bool rows_form(int T, int dtype) { return dtype == SPHATTN_F32 && T > 0 && T <= Low::BQ; }

// Slices of dX's sum there, of 128 ids at least: four waves per CU of 64 columns each, eight where a wave multiplies more than it reads (64 rows,
// 60000 x 1472: 149 us with eight, 200 with four; 17 rows, 50000 x 1024: 57 with four and 5 less for their sum)
int rows_slices(int T, int V, int D)
{
    const int blocks = (D + 63) / 64, most = V / 128 < 128 ? V / 128 : 128, want = ((T > 32 ? 8 : 4) * kCus + blocks - 1) / blocks;
    return most < 1 ? 1 : want < most ? want : most;
}

Vocab vocab_fwd_plan(int T, int V, int D, int dtype, void* workspace)
{
    Vocab p{};
    p.T = T, p.V = V, p.D = D, p.parts = dtype == SPHATTN_F32 ? 2 : 1, p.ld = (int)up_to(D, 8);
    Carve c(workspace);
    p.info = c.take<VocabInfo>(1);
    p.x_exp = c.take<int>(p.parts > 1 ? T : 0);
    p.w_exp = c.take<int>(p.parts > 1 ? up_to(V, 256) : 0);
    p.rows = c.take<int>(T);
    p.place = c.take<int>(T);
    p.target_logit = c.take<float>(T);
    p.partial = c.take<float2>((size_t)((V + 127) / 128) * T);
    p.x = c.take<unsigned short>((size_t)p.parts * T * p.ld);
    // (W and X with rows that the products can read as they are need no copy, but who asks for the size knows no addresses)
    p.w = c.take<unsigned short>((size_t)p.parts * V * p.ld);
    p.bytes = c.used();
    return p;
}

Vocab vocab_bwd_plan(int T, int V, int D, int dtype, void* workspace)
{
    Vocab p{};
    p.T = T, p.V = V, p.D = D, p.parts = dtype == SPHATTN_F32 ? 2 : 1, p.ld = (int)up_to(D, 8);
    const bool few = rows_form(T, dtype);
    p.g_parts = dtype != SPHATTN_F32 ? 1 : few ? 2 : 3;            // (few rows: fp32 as it is)
    const long long row_bytes = 2ll * p.g_parts * (T > 0 ? T : 1);
    size_t limit = (size_t)row_bytes * V <= kOnePieceBytes ? kOnePieceBytes : kPieceBytes;
    if ((size_t)row_bytes * p.ld > limit) limit = (size_t)row_bytes * p.ld;
    long long most = (long long)(limit / row_bytes) / 256 * 256;
    most = most < 256 ? 256 : most > 1 << 18 ? 1 << 18 : most;
    p.n_pieces = (int)((V + most - 1) / most);
    p.piece = (int)up_to((V + p.n_pieces - 1) / p.n_pieces, 256);
    p.n_pieces = (V + p.piece - 1) / p.piece;
    if (few) p.slices = rows_slices(T, V, D);
    else dx_choice(T > 0 ? T : 1, p.ld, p.piece < V ? p.piece : V, p.dx_big, p.slices);
    Carve c(workspace);
    p.info = c.take<VocabInfo>(1);
    p.x_exp = c.take<int>(p.parts > 1 ? T : 0);
    p.w_exp = c.take<int>(p.parts > 1 ? up_to(V, 256) : 0);
    p.rows = c.take<int>(T);
    p.place = c.take<int>(T);
    p.g_target = c.take<int>(T);
    p.g_lse2 = c.take<float>(T);
    p.g = c.take<float>(T);
    p.g_own = c.take<float>(dtype == SPHATTN_F16 ? T : 0);
    p.own_down = c.take<float>(dtype == SPHATTN_F16 ? T : 0);
    p.x = c.take<unsigned short>((size_t)p.parts * T * p.ld);
    p.G = c.take<unsigned short>((size_t)p.g_parts * T * p.piece);
    p.dx = c.take<float>((size_t)p.slices * T * p.ld);
    p.w = c.take<unsigned short>((size_t)p.parts * V * p.ld);
    if (p.g_parts == 3 && T > 0) {
        p.x_sum = c.take<unsigned short>((size_t)3 * T * p.ld);
        p.w_sum = c.take<unsigned short>((size_t)3 * V * p.ld);
    }
    p.bytes = c.used();
    return p;
}

template <class T, Store S, Stage ST>
int launch_tiles(VocabArgs& a, int p, int q, hipStream_t stream)
{
    const auto kern = vocab_tile_kernel<T, S, ST>;
    constexpr int LDS = reads_fp32<T, S, ST>() ? T::WAVES_P * T::BQ * 8 : T::LDS;   // (sums per row only)
    static std::atomic<uint64_t> done{0};
    if (LDS > 65536 && !raise_lds_limit(kern, LDS, done)) return SPHATTN_ERR_LAUNCH;
    a.tiles_p = (p + T::BP - 1) / T::BP;
    const long long tiles = (long long)a.tiles_p * ((q + T::BQ - 1) / T::BQ) * a.slices;
    if (tiles > INT_MAX) return SPHATTN_ERR_SHAPE;
    // (a launch has less than 2^32 threads)
    constexpr long long MOST = 1 << 22;
    for (long long first = 0; first < tiles; first += MOST) {
        a.first = (int)first;
        hipLaunchKernelGGL(kern, dim3((unsigned)(tiles - first < MOST ? tiles - first : MOST)), dim3(T::THREADS), LDS, stream, a);
    }
    return launched();
}

// dX [q,p] and dW [n,p] at once
template <class T, Store S>
int launch_gradients(VocabArgs& dx, VocabArgs& dw, int p, int q, int n, hipStream_t stream)
{
    const auto kern = vocab_gradients_kernel<T, S>;
    static std::atomic<uint64_t> done{0};
    if (T::LDS > 65536 && !raise_lds_limit(kern, T::LDS, done)) return SPHATTN_ERR_LAUNCH;
    dx.tiles_p = dw.tiles_p = (p + T::BP - 1) / T::BP;
    const long long first = (long long)dx.tiles_p * ((q + T::BQ - 1) / T::BQ) * dx.slices, all = first + (long long)dw.tiles_p * ((n + T::BQ - 1) / T::BQ);
    if (all > 1 << 22) {                           // (a launch has less than 2^32 threads)
        const int rc = launch_tiles<T, S, Stage::Dx>(dx, p, q, stream);
        return rc == SPHATTN_OK ? launch_tiles<T, S, Stage::Dw>(dw, p, n, stream) : rc;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)all), dim3(T::THREADS), T::LDS, stream, dx, dw, (int)first);
    return launched();
}

// logits and G: rows decide the tile
template <Store S, Stage ST>
int launch_scores(VocabArgs& a, int V, int T, int& tiles_p, hipStream_t stream)
{
    int rc;
    if (T <= 16) rc = launch_tiles<One, S, ST>(a, V, T, stream);
    else if (S == Store::F32 && T <= 32) rc = launch_tiles<std::conditional_t<S == Store::F32, Few, Low>, S, ST>(a, V, T, stream);
    else if (T <= 64) rc = launch_tiles<Low, S, ST>(a, V, T, stream);
    else if (big_tiles(V, T)) rc = launch_tiles<Big, S, ST>(a, V, T, stream);
    else rc = launch_tiles<Mid, S, ST>(a, V, T, stream);
    tiles_p = a.tiles_p;
    return rc;
}

// whether the products can read rows of D elements at p as they are
bool ready(const void* p, int D, Store S) { return S != Store::F32 && !off(p, 16) && D % 8 == 0; }

RowArgs row_args(const Vocab& p, const void* targets, int id_bytes)
{
    RowArgs r{};
    r.targets = targets, r.id_bytes = id_bytes, r.T = p.T, r.rows = p.rows, r.place = p.place, r.info = p.info;
    return r;
}

// X and W as the products want them; what can be read as it is stays where it is
template <Store S>
void pack(const Vocab& p, const void* X, const void* W, bool pack_x, PackArgs k, Operand& x, Operand& w, hipStream_t stream)
{
    x = Operand{(const unsigned char*)X, 0, p.D * 2, p.T};
    w = Operand{(const unsigned char*)W, 0, p.D * 2, p.V};
    unsigned groups = 0;
    if (pack_x) {
        k.x = PackRows{X, p.x, p.T, p.D, p.ld, (long long)p.T * p.ld, p.x_sum, p.x_exp};
        k.x_groups = (int)(groups = (unsigned)(p.T + kPackRows - 1) / kPackRows);
        x = Operand{(const unsigned char*)p.x, k.x.part * 2, p.ld * 2, p.T};
    }
    if (!ready(W, p.D, S)) {
        k.w = PackRows{W, p.w, p.V, p.D, p.ld, (long long)p.V * p.ld, p.w_sum, p.w_exp};
        groups += (unsigned)(p.V + kPackRows - 1) / kPackRows;
        w = Operand{(const unsigned char*)p.w, k.w.part * 2, p.ld * 2, p.V};
    }
    k.own_rows = p.T <= kOwnRows;
    if (k.compact && !k.own_rows) hipLaunchKernelGGL(vocab_rows_kernel, dim3(1), dim3(kRowsThreads), 0, stream, k.r);
    if (groups) hipLaunchKernelGGL((vocab_pack_kernel<S>), dim3(groups), dim3(kPackThreads), 0, stream, k);
}

template <Store S>
int run_vocab_fwd(const Vocab& p, const void* X, const void* W, const void* targets, int id_bytes, float* losses, float* lse, float* mean,
                  float scale, int reduction, int all_rows, hipStream_t stream)
{
    VocabArgs a{};
    PackArgs k{};
    k.r = row_args(p, targets, id_bytes);
    k.compact = !all_rows && p.T > Low::BQ;        // (up to one tile's rows cost the same whether they count or not)
    if (S == Store::F32 && rows_form(p.T, SPHATTN_F32)) {
        a.P = Operand{(const unsigned char*)W, 0, 0, p.V}, a.Q = Operand{(const unsigned char*)X, 0, 0, p.T};
        a.k = p.D, a.T = p.T;
    } else {
        pack<S>(p, X, W, k.compact || !ready(X, p.D, S), k, a.Q, a.P, stream);
        a.k = p.ld;
        if (S == Store::F32) a.p_exp = p.w_exp, a.q_exp = p.x_exp, a.p_whole = (const float*)W, a.q_whole = (const float*)X, a.D = p.D;
    }
    if (k.compact) a.info = p.info, a.rows = p.rows;
    a.slices = 1, a.V = p.V, a.scale2 = scale * kLog2e;
    a.targets = targets, a.id_bytes = id_bytes;
    a.partial = p.partial, a.partial_ld = p.T, a.target_logit = p.target_logit;
    int tiles = 0;
    const int rc = launch_scores<S, Stage::Logits>(a, p.V, p.T, tiles, stream);
    if (rc != SPHATTN_OK) return rc;
    if (reduction == SPHATTN_LOSS_NONE) mean = nullptr;
    const bool at_once = mean && p.T <= 64 && (long long)tiles * p.T <= 16 * kJoinLossThreads;   // one workgroup, 16 sums per lane at most
    int log_rows = 0;                              // rows of a joining workgroup: half a round of the CUs where they are few
    while (log_rows < 6 && (p.T >> log_rows) > (at_once ? 0 : kCus / 2)) ++log_rows;
    hipLaunchKernelGGL(vocab_join_kernel, dim3((unsigned)(p.T + (1 << log_rows) - 1) >> log_rows), dim3(kJoinLossThreads), 0, stream, p.partial, p.T, tiles,
                       log_rows, p.target_logit, targets, id_bytes, k.compact ? p.place : (const int*)nullptr, all_rows, losses, lse,
                       at_once ? mean : (float*)nullptr, reduction == SPHATTN_LOSS_MEAN, p.T, p.V);
    if (mean && !at_once)
        hipLaunchKernelGGL(vocab_mean_kernel, dim3(1), dim3(1024), 0, stream, losses, targets, id_bytes, p.T, mean, reduction == SPHATTN_LOSS_MEAN);
    return launched();
}

// fp32, at most 64 rows
int run_rows_bwd(const Vocab& p, const void* X, const void* W, PackArgs k, void* dX, void* dW, float scale, hipStream_t stream)
{
    constexpr Store S = Store::F32;
    // which rows count and what G needs of them; no parts are made
    k.x = PackRows{X, nullptr, p.T, p.D, p.ld, 0, nullptr, nullptr};
    k.x_groups = (p.T + kPackRows - 1) / kPackRows, k.own_rows = 1;
    hipLaunchKernelGGL((vocab_pack_kernel<S>), dim3((unsigned)k.x_groups), dim3(kPackThreads), 0, stream, k);
    const int blocks = (p.D + 63) / 64;
    for (int i = 0; i < p.n_pieces; ++i) {
        const int v0 = i * p.piece, n = p.V - v0 < p.piece ? p.V - v0 : p.piece;
        VocabArgs a{};
        a.P = Operand{(const unsigned char*)W + (size_t)v0 * p.D * 4, 0, 0, n}, a.Q = Operand{(const unsigned char*)X, 0, 0, p.T};
        a.info = p.info, a.rows = p.rows, a.k = p.D, a.T = p.T, a.slices = 1, a.V = p.V, a.v0 = v0, a.scale2 = scale * kLog2e;
        a.g_target = p.g_target, a.g_lse2 = p.g_lse2, a.g = p.g, a.G = p.G, a.G_ld = p.piece;
        int tiles;
        const int rc = launch_scores<S, Stage::G>(a, n, p.T, tiles, stream);
        if (rc != SPHATTN_OK) return rc;
        if (dX) {
            a.slices = p.slices, a.out = p.dx, a.out_ld = p.ld, a.accumulate = i > 0;
            const dim3 grid((unsigned)((long long)blocks * p.slices + 3) / 4);
            if (p.T <= 16) hipLaunchKernelGGL((vocab_rows_dx_kernel<1>), grid, dim3(256), 0, stream, a);
            else if (p.T <= 32) hipLaunchKernelGGL((vocab_rows_dx_kernel<2>), grid, dim3(256), 0, stream, a);
            else hipLaunchKernelGGL((vocab_rows_dx_kernel<4>), grid, dim3(256), 0, stream, a);
        }
        if (dW) {
            a.out = (unsigned char*)dW + (size_t)v0 * p.D * 4, a.out_rows = n;
            hipLaunchKernelGGL(vocab_rows_dw_kernel, dim3((unsigned)(((long long)(n + 63) / 64 * blocks + 3) / 4)), dim3(256), 0, stream, a);
        }
    }
    if (dX)
        hipLaunchKernelGGL((vocab_dx_kernel<S>), dim3((unsigned)(p.T + 3) / 4, (unsigned)(p.D + kDxCols - 1) / kDxCols), dim3(256), 0, stream, p.dx, p.slices,
                           p.ld, 128, 1, 0, p.place, p.info, (const float*)nullptr, dX, p.T, p.D);
    return launched();
}

template <Store S>
int run_vocab_bwd(const Vocab& p, const void* X, const void* W, const void* targets, int id_bytes, const float* lse, const float* dloss,
                  void* dX, void* dW, float scale, int reduction, hipStream_t stream)
{
    PackArgs k{};
    k.r = row_args(p, targets, id_bytes);
    k.r.dloss = dloss, k.r.reduce = (Reduce)reduction, k.r.scale = scale, k.r.half = S == Store::F16;
    k.compact = 1, k.lse = lse, k.g_target = p.g_target, k.g_lse2 = p.g_lse2, k.g = p.g;
    // fp16 and one gradient per row: dX's G is scaled row by row, dW's by the largest gradient
    const bool own = S == Store::F16 && reduction == SPHATTN_LOSS_NONE && dX, twice = own && dW;
    if (own) k.g_own = p.g_own, k.own_down = p.own_down;
    Operand x{}, w{};
    if (p.T == 0) {                                // (the info of no rows, which one workgroup writes)
        hipLaunchKernelGGL(vocab_rows_kernel, dim3(1), dim3(kRowsThreads), 0, stream, k.r);
        x = Operand{(const unsigned char*)p.x, 0, p.ld * 2, 0};
    } else if (S == Store::F32 && rows_form(p.T, SPHATTN_F32)) {
        return run_rows_bwd(p, X, W, k, dX, dW, scale, stream);
    } else {
        pack<S>(p, X, W, true, k, x, w, stream);
    }
    int rc = SPHATTN_OK;
    const int dx_tile = p.dx_big ? 256 : 128, dx_at_once = p.dx_big ? kCus : 2 * kCus;
    for (int i = 0; i < p.n_pieces && rc == SPHATTN_OK; ++i) {
        const int v0 = i * p.piece, n = p.V - v0 < p.piece ? p.V - v0 : p.piece;
        const Operand wi{p.T ? w.data + (size_t)v0 * w.ld : nullptr, w.part, w.ld, n};
        // what G is multiplied with: fp32 in parts of its own
        const bool sum_parts = p.x_sum != nullptr;
        const Operand ws = sum_parts ? Operand{(const unsigned char*)(p.w_sum + (size_t)v0 * p.ld), (long long)p.V * p.ld * 2, p.ld * 2, p.ld} : Operand{wi.data, wi.part, wi.ld, p.ld};
        const Operand xs = sum_parts ? Operand{(const unsigned char*)p.x_sum, (long long)p.T * p.ld * 2, p.ld * 2, p.ld} : Operand{x.data, x.part, x.ld, p.ld};
        const Operand G{(const unsigned char*)p.G, (long long)p.T * p.piece * 2, p.piece * 2, 0};
        VocabArgs a{};
        if (S == Store::F32) a.p_exp = p.w_exp + v0, a.q_exp = p.x_exp, a.p_whole = (const float*)W + (size_t)v0 * p.D, a.q_whole = (const float*)X, a.D = p.D, a.rows = p.rows;
        a.P = wi, a.Q = x, a.info = p.info, a.k = p.ld, a.slices = 1, a.V = p.V, a.v0 = v0, a.scale2 = scale * kLog2e;
        a.g_target = p.g_target, a.g_lse2 = p.g_lse2, a.g = own && !twice ? p.g_own : p.g;
        a.G = p.G, a.G_part = (long long)p.T * p.piece, a.G_ld = p.piece;
        int tiles;
        if (p.T > 0) rc = launch_scores<S, Stage::G>(a, n, p.T, tiles, stream);
        if (rc != SPHATTN_OK) break;
        VocabArgs bx{}, bw{};
        const bool with_dx = dX && p.T > 0, with_dw = dW != nullptr;
        bx.P = ws;
        bx.Q = G, bx.Q.size = p.T, bx.info = p.info, bx.k = n, bx.slices = p.slices;
        bx.T = p.T, bx.target = dx_at_once;
        bx.out = p.dx, bx.out_ld = p.ld, bx.out_cols = p.ld, bx.accumulate = i > 0;
        bw.P = xs;
        bw.Q = G, bw.Q.size = (int)up_to(n, 8), bw.info = p.info, bw.slices = 1;
        bw.out = dW ? (unsigned char*)dW + (size_t)v0 * p.D * store_bytes<S>() : nullptr, bw.out_ld = p.D, bw.out_cols = p.D, bw.out_rows = n;
        const bool dw_big = big_tiles(p.ld, n);
        if (twice && p.T > 0) {
            rc = dw_big ? launch_tiles<Big, S, Stage::Dw>(bw, p.ld, n, stream) : launch_tiles<Mid, S, Stage::Dw>(bw, p.ld, n, stream);
            a.g = p.g_own, a.unless_even = 1;
            if (rc == SPHATTN_OK) rc = launch_scores<S, Stage::G>(a, n, p.T, tiles, stream);
            if (rc == SPHATTN_OK) rc = p.dx_big ? launch_tiles<Big, S, Stage::Dx>(bx, p.ld, p.T, stream) : launch_tiles<Mid, S, Stage::Dx>(bx, p.ld, p.T, stream);
            continue;
        }
        if (with_dx && with_dw && !p.dx_big && !dw_big) {
            rc = launch_gradients<Mid, S>(bx, bw, p.ld, p.T, n, stream);
            continue;
        }
        if (with_dx) rc = p.dx_big ? launch_tiles<Big, S, Stage::Dx>(bx, p.ld, p.T, stream) : launch_tiles<Mid, S, Stage::Dx>(bx, p.ld, p.T, stream);
        if (rc == SPHATTN_OK && with_dw)
            rc = dw_big ? launch_tiles<Big, S, Stage::Dw>(bw, p.ld, n, stream) : launch_tiles<Mid, S, Stage::Dw>(bw, p.ld, n, stream);
    }
    if (rc == SPHATTN_OK && dX && p.T > 0)
        hipLaunchKernelGGL((vocab_dx_kernel<S>), dim3((unsigned)(p.T + 3) / 4, (unsigned)(p.D + kDxCols - 1) / kDxCols), dim3(256), 0, stream, p.dx, p.slices, p.ld,
                           dx_tile, (p.ld + dx_tile - 1) / dx_tile, dx_at_once, p.place, p.info, own ? p.own_down : (const float*)nullptr, dX, p.T, p.D);
    return rc == SPHATTN_OK ? launched() : rc;
}

int vocab_check(const void* X, const void* W, const void* targets, int id_bytes, int T, int V, int D, float scale, int reduction, int dtype)
{
    if (!vocab_shape(T, V, D)) return SPHATTN_ERR_SHAPE;
    if (!element_bytes(dtype) || (id_bytes != 4 && id_bytes != 8)) return SPHATTN_ERR_DTYPE;
    if (!W || (T > 0 && (!X || !targets))) return SPHATTN_ERR_NULL;
    if (off(X, element_bytes(dtype)) || off(W, element_bytes(dtype)) || off(targets, id_bytes)) return SPHATTN_ERR_ALIGN;
    if (!std::isfinite(scale) || reduction < SPHATTN_LOSS_NONE || reduction > SPHATTN_LOSS_MEAN) return SPHATTN_ERR_VALUE;
    return SPHATTN_OK;
}

}  // namespace

extern "C" {

int sphattn_embed_fwd(const void* tokens, int id_bytes, const void* table, const float* mult, void* O,
                      int T, int V, int D, float scale, int dtype, void* stream)
{
    const int rc = embed_check(tokens, id_bytes, mult, T, V, D, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (!table || (T > 0 && !O)) return SPHATTN_ERR_NULL;
    const size_t e = (size_t)element_bytes(dtype);
    if (off(table, e) || off(O, e)) return SPHATTN_ERR_ALIGN;
    const Range written[] = {{O, (size_t)T * D * e}};
    const Range read[] = {{tokens, (size_t)T * id_bytes}, {table, (size_t)V * D * e}, {mult, mult ? (size_t)T * 4 : 0}};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    if (T == 0) return SPHATTN_OK;
    const hipStream_t s = (hipStream_t)stream;
    switch (dtype) {
    case SPHATTN_F32: return run_embed_fwd<Store::F32>(tokens, id_bytes, table, mult, O, T, V, D, scale, s);
    case SPHATTN_BF16: return run_embed_fwd<Store::Bf16>(tokens, id_bytes, table, mult, O, T, V, D, scale, s);
    default: return run_embed_fwd<Store::F16>(tokens, id_bytes, table, mult, O, T, V, D, scale, s);
    }
}

size_t sphattn_embed_bwd_workspace_bytes(int T, int V, int D)
{
    return embed_shape(T, V, D) ? embed_plan(T, V, D, nullptr).bytes : 0;
}

int sphattn_embed_bwd(const void* tokens, int id_bytes, const float* mult, const void* dO, void* dtable,
                      int T, int V, int D, float scale, int dtype,
                      void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = embed_check(tokens, id_bytes, mult, T, V, D, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (!dtable || (T > 0 && !dO)) return SPHATTN_ERR_NULL;
    const size_t e = (size_t)element_bytes(dtype);
    if (off(dtable, e) || off(dO, e)) return SPHATTN_ERR_ALIGN;
    const EmbedPlan p = embed_plan(T, V, D, workspace);
    if (!workspace || off(workspace, 16) || workspace_bytes < p.bytes) return SPHATTN_ERR_WORKSPACE;
    const Range written[] = {{dtable, (size_t)V * D * e}, {workspace, p.bytes}};
    const Range read[] = {{tokens, (size_t)T * id_bytes}, {dO, (size_t)T * D * e}, {mult, mult ? (size_t)T * 4 : 0}};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    const hipStream_t s = (hipStream_t)stream;
    switch (dtype) {
    case SPHATTN_F32: return run_embed_bwd<Store::F32>(p, tokens, id_bytes, mult, dO, dtable, T, V, D, scale, s);
    case SPHATTN_BF16: return run_embed_bwd<Store::Bf16>(p, tokens, id_bytes, mult, dO, dtable, T, V, D, scale, s);
    default: return run_embed_bwd<Store::F16>(p, tokens, id_bytes, mult, dO, dtable, T, V, D, scale, s);
    }
}

size_t sphattn_vocab_loss_workspace_bytes(int T, int V, int D, int dtype)
{
    return vocab_shape(T, V, D) && element_bytes(dtype) ? vocab_fwd_plan(T, V, D, dtype, nullptr).bytes : 0;
}

int sphattn_vocab_loss_fwd(const void* X, const void* W, const void* targets, int id_bytes,
                           float* losses, float* lse, float* mean,
                           int T, int V, int D, float scale, int reduction, int all_rows, int dtype,
                           void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = vocab_check(X, W, targets, id_bytes, T, V, D, scale, reduction, dtype);
    if (rc != SPHATTN_OK) return rc;
    if (T > 0 && !losses) return SPHATTN_ERR_NULL;
    if (off(losses, 4) || off(lse, 4) || off(mean, 4)) return SPHATTN_ERR_ALIGN;
    const size_t e = (size_t)element_bytes(dtype);
    const Vocab p = vocab_fwd_plan(T, V, D, dtype, workspace);
    if (!workspace || off(workspace, 16) || workspace_bytes < p.bytes) return SPHATTN_ERR_WORKSPACE;
    const Range written[] = {{losses, (size_t)T * 4}, {lse, lse ? (size_t)T * 4 : 0}, {mean, mean ? (size_t)4 : 0}, {workspace, p.bytes}};
    const Range read[] = {{X, (size_t)T * D * e}, {W, (size_t)V * D * e}, {targets, (size_t)T * id_bytes}};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    const hipStream_t s = (hipStream_t)stream;
    if (T == 0) {
        if (mean && reduction != SPHATTN_LOSS_NONE)
            hipLaunchKernelGGL(vocab_mean_kernel, dim3(1), dim3(1024), 0, s, losses, targets, id_bytes, 0, mean, 0);
        return launched();
    }
    switch (dtype) {
    case SPHATTN_F32: return run_vocab_fwd<Store::F32>(p, X, W, targets, id_bytes, losses, lse, mean, scale, reduction, all_rows, s);
    case SPHATTN_BF16: return run_vocab_fwd<Store::Bf16>(p, X, W, targets, id_bytes, losses, lse, mean, scale, reduction, all_rows, s);
    default: return run_vocab_fwd<Store::F16>(p, X, W, targets, id_bytes, losses, lse, mean, scale, reduction, all_rows, s);
    }
}

size_t sphattn_vocab_loss_bwd_workspace_bytes(int T, int V, int D, int dtype)
{
    return vocab_shape(T, V, D) && element_bytes(dtype) ? vocab_bwd_plan(T, V, D, dtype, nullptr).bytes : 0;
}

int sphattn_vocab_loss_bwd(const void* X, const void* W, const void* targets, int id_bytes,
                           const float* lse, const float* dloss, void* dX, void* dW,
                           int T, int V, int D, float scale, int reduction, int dtype,
                           void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = vocab_check(X, W, targets, id_bytes, T, V, D, scale, reduction, dtype);
    if (rc != SPHATTN_OK) return rc;
    if ((T > 0 && (!lse || !dloss)) || (!dX && !dW)) return SPHATTN_ERR_NULL;
    const size_t e = (size_t)element_bytes(dtype);
    if (off(lse, 4) || off(dloss, 4) || off(dX, e) || off(dW, e)) return SPHATTN_ERR_ALIGN;
    const Vocab p = vocab_bwd_plan(T, V, D, dtype, workspace);
    if (!workspace || off(workspace, 16) || workspace_bytes < p.bytes) return SPHATTN_ERR_WORKSPACE;
    const Range written[] = {{dX, (size_t)T * D * e}, {dW, (size_t)V * D * e}, {workspace, p.bytes}};
    const Range read[] = {{X, (size_t)T * D * e}, {W, (size_t)V * D * e}, {targets, (size_t)T * id_bytes}, {lse, (size_t)T * 4},
                          {dloss, reduction == SPHATTN_LOSS_NONE ? (size_t)T * 4 : 4}};
    if (any_meet(written, read)) return SPHATTN_ERR_ALIAS;
    const hipStream_t s = (hipStream_t)stream;
    switch (dtype) {
    case SPHATTN_F32: return run_vocab_bwd<Store::F32>(p, X, W, targets, id_bytes, lse, dloss, dX, dW, scale, reduction, s);
    case SPHATTN_BF16: return run_vocab_bwd<Store::Bf16>(p, X, W, targets, id_bytes, lse, dloss, dX, dW, scale, reduction, s);
    default: return run_vocab_bwd<Store::F16>(p, X, W, targets, id_bytes, lse, dloss, dX, dW, scale, reduction, s);
    }
}

size_t sphattn_clip_grads_workspace_bytes(int n)
{
    return n < 0 ? 0 : (((size_t)n + kClipBatch - 1) / kClipBatch + (n == 0)) * kClipMostGroups * sizeof(double);
}

int sphattn_clip_grads(const void* const* in, void* const* out, const long long* size, const int* dtype, int n,
                       float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream)
{
    if (n < 0) return SPHATTN_ERR_SHAPE;
    if (!norm || (n > 0 && (!in || !out || !size || !dtype))) return SPHATTN_ERR_NULL;
    if (off(norm, 4)) return SPHATTN_ERR_ALIGN;
    if (!(max_norm >= 0.f)) return SPHATTN_ERR_VALUE;
    long long elements = 0;
    for (int i = 0; i < n; ++i) {
        const int e = element_bytes(dtype[i]);
        if (!e) return SPHATTN_ERR_DTYPE;
        if (size[i] < 0 || size[i] > kClipMostElements - elements) return SPHATTN_ERR_SHAPE;
        elements += size[i];
        if (size[i] > 0 && (!in[i] || !out[i])) return SPHATTN_ERR_NULL;
        if (off(in[i], e) || off(out[i], e)) return SPHATTN_ERR_ALIGN;
        const Range a{in[i], (size_t)size[i] * e}, b{out[i], a.bytes};
        if ((in[i] != out[i] && meet(a, b)) || meet(a, {norm, 4}) || meet(b, {norm, 4}) || meet(b, {workspace, workspace_bytes}) || meet(a, {workspace, workspace_bytes}))
            return SPHATTN_ERR_ALIAS;
    }
    if (!workspace || off(workspace, 16) || workspace_bytes < sphattn_clip_grads_workspace_bytes(n)) return SPHATTN_ERR_WORKSPACE;
    if (meet({norm, 4}, {workspace, workspace_bytes})) return SPHATTN_ERR_ALIAS;

    const hipStream_t s = (hipStream_t)stream;
    double* sums = (double*)workspace;
    ClipList list;
    auto fill = [&](int i0) {
        list.chunks = 0;
        for (int j = 0; j < kClipBatch; ++j) {
            const int i = i0 + j;
            list.first[j] = i < n ? (int)list.chunks : INT_MAX;
            if (i >= n) continue;
            list.in[j] = in[i], list.out[j] = out[i], list.size[j] = size[i];
            const Store t = dtype[i] == SPHATTN_F32 ? Store::F32 : dtype[i] == SPHATTN_BF16 ? Store::Bf16 : Store::F16;
            list.type[j] = (unsigned char)((int)t | (off(in[i], 16) || off(out[i], 16) ? 0 : 128));
            list.chunks += (size[i] + kClipChunk - 1) / kClipChunk;
        }
    };
    auto groups_of = [](long long chunks) { return (int)(chunks < 1 ? 1 : chunks < kClipMostGroups ? chunks : kClipMostGroups); };
    int n_sums = 0;
    for (int i = 0; i < n || i == 0; i += kClipBatch) {
        fill(i);
        const int groups = groups_of(list.chunks);
        hipLaunchKernelGGL(clip_squares_kernel, dim3((unsigned)groups), dim3(kClipThreads), 0, s, list, sums + n_sums);
        n_sums += groups;
    }
    // (backwards, also within a launch: what was read last is in the last-level cache still)
    for (int i = n > 0 ? (n - 1) / kClipBatch * kClipBatch : 0; i >= 0; i -= kClipBatch) {
        if (n > kClipBatch) fill(i);
        const int groups = groups_of(list.chunks);
        hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)groups), dim3(kClipThreads), 0, s, list, sums, n_sums, max_norm, norm, i == 0);
    }
    return launched();
}

}  // extern "C"
