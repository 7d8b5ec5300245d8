// Embedding lookup with scaling, y[i] = scale * table[tokens[i]], and the gradient of its table, dtable[v] = scale * sum of the dy rows whose token is v.
// Both move rows of C values and do next to nothing with them: the bound is HBM (lookup: rows read and written; gradient: dy read, the table's
// gradient written, zeros included).
//
// The gradient's sums are made in the order of the tokens' positions (in pieces of fixed size), never by atomic additions, so that equal inputs give equal bits.
// Few tokens: a warp per token looks through all of them.  Otherwise the positions are sorted by token (stable) and the sorted list is cut into tiles:
//   sort    every CTA owns a share of the table's rows: it picks their tokens out of all (and counts those of the CTAs in front, so it knows its place in the
//           list without asking anyone), sorts them, and fills the rows that none names with zeros.  Reading all tokens in every CTA costs 1 us per 8000;
//           a cluster that sorted for all took 56 us for 131072 tokens, this 28.  (All rows filled from the start, beside the sort: 112 instead of 104 us for
//           131072 rows of 1024, of which 46000 occur; HBM takes writes alone at 4.8 to 5.5 TB/s, so those that are written anyway are better left out.)
//   sums    a team of threads per tile adds the rows up, and writes a token's sum when the next one begins; a sum that began in an earlier tile is left as
//           a partial row
//   joins   the team of the tile in which a token began adds the partial rows of the following tiles to its row
#include "seqops.h"
#include "launch.h"

#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

namespace fdg {
namespace {

using bf16 = __nv_bfloat16;

// ---- vectors of N values
template <int B> struct Word;
template <> struct Word<16> { using W = uint4; };
template <> struct Word<8> { using W = uint2; };
template <> struct Word<4> { using W = unsigned; };
template <> struct Word<2> { using W = unsigned short; };
template <typename T, int N> using Raw = typename Word<sizeof(T) * N>::W;
template <typename T, int N> __device__ __forceinline__ void unpack(const Raw<T, N>& r, float (&x)[N]) {
    const T* const p = (const T*)&r;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)p[i];
}
template <typename T, int N> __device__ __forceinline__ Raw<T, N> pack(const float (&x)[N]) {
    Raw<T, N> r;
    T* const p = (T*)&r;
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = (T)x[i];
    return r;
}

// ---- lookup: every thread moves UNROLL vectors of the output, neighbours side by side.  It divides once (256 vectors on are row_step rows and col_step vectors on):
// 16384 x 1024 bf16 10.4 us, 10.7 with a division per vector; what is left are two loads in a row and the launch.
constexpr int UNROLL = 4;
template <typename T, int N>
__global__ void __launch_bounds__(256) embed_fwd_k(const int32_t* __restrict__ tokens, unsigned n, const T* __restrict__ table, unsigned vocab, int C, unsigned per_row, unsigned row_step,
                                                   unsigned col_step, float scale, T* __restrict__ y, long ys) {
    const long first = (long)blockIdx.x * (256 * UNROLL) + threadIdx.x;
    unsigned row0 = first >> 32 ? (unsigned)(first / per_row) : (unsigned)first / per_row, c = (unsigned)first - row0 * per_row;
    Raw<T, N> r[UNROLL];
    unsigned row[UNROLL], col[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        row[u] = row0; col[u] = c * N;
        r[u] = Raw<T, N>{};
        if (row0 < n) {
            const unsigned tok = (unsigned)tokens[row0];                 // negative ids are large ones
            if (tok < vocab) r[u] = *(const Raw<T, N>*)(table + (long)tok * C + col[u]);
        }
        row0 += row_step; c += col_step;
        if (c >= per_row) { c -= per_row; ++row0; }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        if (row[u] >= n) continue;
        float x[N];
        unpack<T, N>(r[u], x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= scale;
        *(Raw<T, N>*)(y + (long)row[u] * ys + col[u]) = pack<T, N>(x);
    }
}

// Zeros to those of `rows` rows of dtable that none of n tokens names, by a CTA of THREADS.  token(i): the row of token i, counted from 0 (negative or behind: not one of these);
// place(r): where row r is in dtable, at or behind vocab: nowhere.  Written rows are the bound, so those that the sums write are left out: the CTA marks the rows that occur.
constexpr int FILL_ROWS = 8192;                 // that it looks at a time
template <int THREADS, typename Tokens, typename Place>
__device__ __forceinline__ void fill_rows(Tokens token, int n, float* dtable, long rows, long vocab, Place place, int C, bool vec, unsigned* named) {
    for (long b = 0; b < rows; b += FILL_ROWS) {
        const int now = (int)min((long)FILL_ROWS, rows - b);
        __syncthreads();
        for (int i = threadIdx.x; i < (now + 31) / 32; i += THREADS) named[i] = 0;
        __syncthreads();
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += THREADS) {
            const long t = token(i) - b;                        // (common tokens: one atomic operation, not thousands at one address)
            if (t >= 0 && t < now && !(((volatile unsigned*)named)[t >> 5] >> (t & 31) & 1)) atomicOr(&named[t >> 5], 1u << (t & 31));
        }
        __syncthreads();
        const unsigned per = vec ? C / 4 : C;
        unsigned row = threadIdx.x / per, col = threadIdx.x - row * per;
        const unsigned row_step = THREADS / per, col_step = THREADS - row_step * per;
#pragma unroll 4
        for (; row < (unsigned)now;) {
            const long at = place(b + row);
            if (at < vocab && !(named[row >> 5] >> (row & 31) & 1)) {
                float* const d = dtable + at * C;
                if (vec) ((float4*)d)[col] = make_float4(0.f, 0.f, 0.f, 0.f); else d[col] = 0.f;
            }
            row += row_step; col += col_step;
            if (col >= per) { col -= per; ++row; }
        }
    }
}

// ---- gradient of few tokens, in one launch
// Sorted, 512 ids of 32000 x 1024 take 38 us instead of 26 (1000 x 128: 17 instead of 6), 2048 take 39 instead of 38; the more equal ones there are, the longer a warp adds: where three in
// ten are one id, 512 take 60 (27), sorted 37 (17).  (Which ids there are is not known on the host; the line is for ids that mostly differ.)
constexpr int FEW = 512;
// CTAs 0 .. sum_ctas - 1: a warp per token and 32 N channels; it goes on if no earlier token is the same, and adds up all that are, in order.  The
// others fill the rows that no token names.
template <typename T, int N>
__global__ void __launch_bounds__(256) embed_few_k(const int32_t* __restrict__ tokens, int n, const T* __restrict__ dy, long dys, long vocab, int C, int slices, float scale,
                                                   int accum, float* __restrict__ dtable, int sum_ctas) {
    __shared__ int tok_[FEW];
    __shared__ unsigned named[FILL_ROWS / 32];
#pragma unroll
    for (int i = 0; i < FEW; i += 256) if (i + threadIdx.x < n) tok_[i + threadIdx.x] = tokens[i + threadIdx.x];
    __syncthreads();
    if ((int)blockIdx.x >= sum_ctas) {
        const long ctas = gridDim.x - sum_ctas, per = (vocab + ctas - 1) / ctas, r0 = (blockIdx.x - sum_ctas) * per;
        fill_rows<256>([&](int i) { return (long)tok_[i] - r0; }, n, dtable, min(vocab - r0, per), vocab, [&](long r) { return r0 + r; }, C, N > 2, named);
        return;
    }
    const int warp = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, i = warp / slices, c = (warp - i * slices) * 32 * N + lane * N;
    if (i >= n) return;
    const int tok = tok_[i];
    if (tok < 0 || tok >= vocab) return;
    bool same = false;
    for (int j = lane; j < i; j += 32) same |= tok_[j] == tok;
    if (__any_sync(~0u, same)) return;
    const bool in = c < C;
    float sum[N] = {};
    for (int j = i; j < n; j += 32) {
        unsigned hits = __ballot_sync(~0u, j + lane < n && tok_[j + lane] == tok);
        auto add = [&](const Raw<T, N>& row) {
            float x[N];
            unpack<T, N>(row, x);
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] += x[k];
        };
        if (hits == ~0u) {                                      // one id everywhere
            if (in)
                for (int q = 0; q < 32; q += 16) {
                    Raw<T, N> r[16];
#pragma unroll
                    for (int u = 0; u < 16; ++u) r[u] = *(const Raw<T, N>*)(dy + (long)(j + q + u) * dys + c);
#pragma unroll
                    for (int u = 0; u < 16; ++u) add(r[u]);
                }
            hits = 0;
        }
        while (hits) {
            Raw<T, N> r[4];
            int m = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (hits) { const int q = __ffs(hits) - 1; hits &= hits - 1; m = u + 1; if (in) r[u] = *(const Raw<T, N>*)(dy + (j + q) * dys + c); }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u < m && in) add(r[u]);
        }
    }
    if (!in) return;
    float* const d = dtable + (long)tok * C + c;
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] = accum ? fmaf(sum[k], scale, d[k]) : sum[k] * scale;
}

// ---- gradient of many tokens
constexpr int SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32, MAX_BITS = 10;
constexpr int OWNER_BITS = 7, OWNERS = 1 << OWNER_BITS;

// the lanes whose d is this one's, by ballots: __match_any_sync takes longer for 32 different values (a sort 89 us instead of 56)
__device__ __forceinline__ unsigned equals(unsigned d, int bits) {
    unsigned m = ~0u;
    for (int b = 0; b < bits; ++b) { const bool on = d >> b & 1; const unsigned v = __ballot_sync(~0u, on); m &= on ? v : ~v; }
    return m;
}

// A CTA owns every 128th group of 2^gs rows of the table: frequent tokens often have small ids, and with a range each (128 times as many rows in a row) the first CTA would sort most of
// them: 131072 ids whose frequency falls like 1 / id, 131072 rows of 1024, 219 us instead of 378; a million, 32000 rows of 64, 382 instead of 1183.  An owner's rows are counted from 0.
__device__ __forceinline__ unsigned owner_of(unsigned token, int gs) { return token >> gs & (OWNERS - 1); }
__device__ __forceinline__ unsigned row_in(unsigned token, int gs) { return token >> (OWNER_BITS + gs) << gs | (token & ((1u << gs) - 1)); }
__device__ __forceinline__ long row_of(unsigned row, unsigned owner, int gs) { return ((long)(row >> gs) << OWNER_BITS | owner) << gs | (row & ((1u << gs) - 1)); }

// The list: entries {token, position} by owner, then token, then position; tokens outside the table are not in it.  *count: its length.
__global__ void __launch_bounds__(SORT_THREADS, 1) embed_sort_k(const int32_t* __restrict__ tokens, int n, unsigned vocab, uint2* list, uint2* other, int rows, int gs, int passes, int bits,
                                                               float* dtable, int C, int vec, unsigned* count, unsigned* chains) {
    extern __shared__ unsigned hist[];                          // [warp][bin]
    __shared__ unsigned sums[SORT_WARPS], less[SORT_WARPS];
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned self = blockIdx.x;
    auto is_mine = [&](unsigned t) { return t < vocab && owner_of(t, gs) == self; };
    auto is_less = [&](unsigned t) { return t < vocab && owner_of(t, gs) < self; };
    const bool aligned = (uintptr_t)tokens % 16 == 0;
    // tokens of the warp, 128 at a time, four consecutive ones a lane, to f(first position, the four)
    const int per_warp = (int)(((n + SORT_WARPS - 1l) / SORT_WARPS + 127) / 128 * 128);
    const int begin = (int)min((long)n, (long)w * per_warp), end = (int)min((long)n, (long)(w + 1) * per_warp);
    auto each = [&](auto f) {
        constexpr int AHEAD = 4;
        for (int i0 = begin; i0 < end; i0 += 128 * AHEAD) {
            uint4 t[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int i = i0 + u * 128 + lane * 4;
                if (aligned && i + 3 < end) t[u] = *(const uint4*)(tokens + i);
                else t[u] = make_uint4(i < end ? tokens[i] : ~0u, i + 1 < end ? tokens[i + 1] : ~0u, i + 2 < end ? tokens[i + 2] : ~0u, i + 3 < end ? tokens[i + 3] : ~0u);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) if (i0 + u * 128 < end) f(i0 + u * 128 + lane * 4, t[u]);
        }
    };
    // how many have an earlier owner, how many are the warp's of this one
    unsigned mine = 0, smaller = 0;
    each([&](int, const uint4& t) {
        mine += is_mine(t.x) + is_mine(t.y) + is_mine(t.z) + is_mine(t.w);
        smaller += is_less(t.x) + is_less(t.y) + is_less(t.z) + is_less(t.w);
    });
    mine = __reduce_add_sync(~0u, mine); smaller = __reduce_add_sync(~0u, smaller);
    if (lane == 0) { sums[w] = mine; less[w] = smaller; }
    __syncthreads();
    unsigned at = 0, m = 0, base = 0;                           // the warp's place, the owner's entries, its place in the list
    for (int q = 0; q < SORT_WARPS; ++q) { if (q < w) at += sums[q]; m += sums[q]; base += less[q]; }
    if (threadIdx.x == 0) {
        if (self == gridDim.x - 1) *count = base + m;
        if (blockIdx.x == 0) *chains = 0;
    }
    // the owner's entries, in order
    uint2* src = (passes & 1 ? other : list) + base;
    uint2* dst = (passes & 1 ? list : other) + base;
    each([&](int i, const uint4& t) {
        const bool a = is_mine(t.x), b = is_mine(t.y), c = is_mine(t.z), d = is_mine(t.w);
        if (!__any_sync(~0u, a || b || c || d)) return;
        const unsigned A = __ballot_sync(~0u, a), B = __ballot_sync(~0u, b), Cc = __ballot_sync(~0u, c), D = __ballot_sync(~0u, d), lt = (1u << lane) - 1;
        unsigned to = at + __popc(A & lt) + __popc(B & lt) + __popc(Cc & lt) + __popc(D & lt);
        if (a) src[to++] = make_uint2(t.x, i);
        if (b) src[to++] = make_uint2(t.y, i + 1);
        if (c) src[to++] = make_uint2(t.z, i + 2);
        if (d) src[to++] = make_uint2(t.w, i + 3);
        at += __popc(A) + __popc(B) + __popc(Cc) + __popc(D);
    });
    __syncthreads();
    // sorted by `bits` bits of the owner's row a pass; a warp has a run of the entries and counts of its own, and AHEAD times 32 of them on their way
    const int bins = 1 << bits, run = (int)((m + SORT_THREADS - 1) / SORT_THREADS * 32);
    const int lo = (int)min((long)m, (long)w * run), hi = (int)min((long)m, (long)(w + 1) * run);
    unsigned* const own = hist + w * bins;
    constexpr int AHEAD = 4;
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        for (int i = threadIdx.x; i < SORT_WARPS * bins; i += SORT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i0 = lo; i0 < hi; i0 += 32 * AHEAD) {
            unsigned t[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) { const int i = i0 + u * 32 + lane; t[u] = i < hi ? __ldcg(&src[i].x) : 0; }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int i = i0 + u * 32;
                if (i >= hi) break;
                const bool in = i + lane < hi;
                const unsigned d = row_in(t[u], gs) >> shift & (bins - 1), peers = equals(d, bits) & __ballot_sync(~0u, in);
                if (in && lane == __ffs(peers) - 1) own[d] += __popc(peers);
                __syncwarp();
            }
        }
        __syncthreads();
        // where every warp's part of every bin begins
        unsigned all = 0;
        const int b = threadIdx.x;
        if (b < bins)
#pragma unroll 8
            for (int q = 0; q < SORT_WARPS; ++q) { const unsigned t = hist[q * bins + b]; hist[q * bins + b] = all; all += t; }
        unsigned scan = all;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) { const unsigned t = __shfl_up_sync(~0u, scan, d); if (lane >= d) scan += t; }
        if (lane == 31) sums[w] = scan;
        __syncthreads();
        unsigned before = scan - all;
        for (int q = 0; q < w; ++q) before += sums[q];
        if (b < bins)
#pragma unroll 8
            for (int q = 0; q < SORT_WARPS; ++q) hist[q * bins + b] += before;
        __syncthreads();
        for (int i0 = lo; i0 < hi; i0 += 32 * AHEAD) {
            uint2 e[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) { const int i = i0 + u * 32 + lane; e[u] = i < hi ? __ldcg(src + i) : make_uint2(0, 0); }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int i = i0 + u * 32;
                if (i >= hi) break;
                const bool in = i + lane < hi;
                const unsigned d = row_in(e[u].x, gs) >> shift & (bins - 1), peers = equals(d, bits) & __ballot_sync(~0u, in), to = own[d];
                __syncwarp();
                if (in) {
                    if (lane == __ffs(peers) - 1) own[d] = to + __popc(peers);
                    dst[to + __popc(peers & ((1u << lane) - 1))] = e[u];
                }
                __syncwarp();
            }
        }
        __syncthreads();
        uint2* const t = src; src = dst; dst = t;
    }
    if (dtable) fill_rows<SORT_THREADS>([&](int i) { return (long)row_in(__ldcg(&src[i].x), gs); }, (int)m, dtable, rows, vocab, [&](long r) { return row_of((unsigned)r, self, gs); }, C, vec, hist);
}

// How the sorted list is cut: tiles of `tile` entries, each summed by teams of `tx` threads (of which `slices` cover the channels).
struct Plan { int tx, slices, tile, tiles; };
// What the sums leave for the joins.
struct Left {
    float* part;            // [tile][C]: sums of the tokens that began in an earlier tile
    int* head;              // [tile]: that token, or -1
    unsigned* count;        // entries of the list
    unsigned* chains;       // how many tokens go on behind the tile in which they began,
    int2* chain;            // and these tiles and tokens, in any order
};

constexpr int BATCH = 8;                        // rows on their way at once (with whole vectors 80 registers do not quite hold them: 20 and 28 bytes a thread, fp32 and bf16, are spilled)
template <typename T, int N>
__global__ void __launch_bounds__(256, 3) embed_sums_k(const uint2* __restrict__ list, const T* __restrict__ dy, long dys, int C, float scale, int accum,
                                                    float* __restrict__ dtable, Left left, Plan p) {
    const int tile = blockIdx.x * (256 / p.tx) + threadIdx.x / p.tx;
    const int c = (blockIdx.y * p.tx + threadIdx.x % p.tx) * N;
    const int n = (int)*left.count, t0 = tile * p.tile, t1 = min(n, t0 + p.tile);
    if (tile >= p.tiles || c >= C) return;
    if (t0 >= n) {                                              // (tokens outside the table have shortened the list)
        if (c == 0) left.head[tile] = -1;
        return;
    }
    unsigned now = list[t0].x;
    bool begun = t0 > 0 && list[t0 - 1].x == now;               // in an earlier tile
    if (c == 0) {
        left.head[tile] = begun ? (int)now : -1;
        if (t1 < n) {                                           // the last token of the tile goes on, and began here
            const unsigned last = list[t1 - 1].x;
            if (list[t1].x == last && !(begun && last == now)) left.chain[atomicAdd(left.chains, 1u)] = make_int2(tile, (int)last);
        }
    }
    float sum[N] = {};
    auto leave = [&]() {
        float* const d = begun ? left.part + (long)tile * C + c : dtable + (long)now * C + c;
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] = begun ? sum[k] : accum ? fmaf(sum[k], scale, d[k]) : sum[k] * scale;
        if constexpr (N >= 4) {                                 // (rows of such tables start on 16 bytes)
#pragma unroll
            for (int k = 0; k < N; k += 4) *(float4*)(d + k) = make_float4(sum[k], sum[k + 1], sum[k + 2], sum[k + 3]);
        } else
#pragma unroll
            for (int k = 0; k < N; ++k) d[k] = sum[k];
    };
    for (int i = t0; i < t1; i += BATCH) {
        unsigned key[BATCH];
        Raw<T, N> r[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (i + u >= t1) continue;
            const uint2 e = list[i + u];
            key[u] = e.x;
            r[u] = *(const Raw<T, N>*)(dy + (long)e.y * dys + c);
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (i + u >= t1) break;
            if (key[u] != now) {
                leave();
                now = key[u]; begun = false;
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] = 0.f;
            }
            float x[N];
            unpack<T, N>(r[u], x);
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] += x[k];
        }
    }
    leave();
}

// A CTA per such token and JOIN_TX threads' channels, of 4 (N = 4, rows on 16 bytes) or one: its groups of threads add equal runs of the tiles that follow, then the groups are
// added in order.
constexpr int JOIN_TX = 64, JOIN_GROUPS = 256 / JOIN_TX, JOIN_BATCH = 8;
template <int N>
__global__ void __launch_bounds__(256) embed_joins_k(int C, float scale, float* __restrict__ dtable, Left left, Plan p) {
    __shared__ float sums[JOIN_GROUPS][JOIN_TX * N];
    const int c = (blockIdx.y * JOIN_TX + threadIdx.x % JOIN_TX) * N, group = threadIdx.x / JOIN_TX;
    const unsigned* const chains = left.chains;
    int2 next = left.chain[blockIdx.x];                         // (whether it is one of them or not: the loads wait for nothing)
    const int all = (int)*chains;
    for (int e = blockIdx.x; e < all; e += gridDim.x) {
        const int first = next.x + 1, now = next.y;
        if (e + (int)gridDim.x < all) next = left.chain[e + gridDim.x];
        float* const d = dtable + (long)now * C + c;
        Raw<float, N> old{};
        if (group == 0 && c < C) {
            float x[N];
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = d[k];
            old = pack<float, N>(x);
        }
        int length = 0;                                         // tiles that it goes on through
        for (int j = first;; j += 256) {
            const int more = __syncthreads_count(j + (int)threadIdx.x < p.tiles && left.head[j + threadIdx.x] == now);
            length += more;
            if (more < 256) break;
        }
        const int run = (length + JOIN_GROUPS - 1) / JOIN_GROUPS, lo = first + group * run, hi = min(first + length, lo + run);
        float sum[N] = {};
        if (c < C)
            for (int j = lo; j < hi; j += JOIN_BATCH) {
                Raw<float, N> v[JOIN_BATCH];
#pragma unroll
                for (int u = 0; u < JOIN_BATCH; ++u) if (j + u < hi) v[u] = *(const Raw<float, N>*)(left.part + (long)(j + u) * C + c);
#pragma unroll
                for (int u = 0; u < JOIN_BATCH; ++u)
                    if (j + u < hi) {
                        float x[N];
                        unpack<float, N>(v[u], x);
#pragma unroll
                        for (int k = 0; k < N; ++k) sum[k] += x[k];
                    }
            }
#pragma unroll
        for (int k = 0; k < N; ++k) sums[group][threadIdx.x % JOIN_TX * N + k] = sum[k];
        __syncthreads();
        if (group == 0 && c < C) {
            float x[N];
            unpack<float, N>(old, x);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float t = sum[k];
#pragma unroll
                for (int q = 1; q < JOIN_GROUPS; ++q) t += sums[q][threadIdx.x * N + k];
                d[k] = fmaf(t, scale, x[k]);
            }
        }
    }
}

// elements that may be moved at once: 16 bytes' worth, 2, or 1
template <typename T> int vector(const void* a, long stride_a, long C) {
    for (int n : {16 / (int)sizeof(T), 2}) if ((uintptr_t)a % (n * sizeof(T)) == 0 && stride_a % n == 0 && C % n == 0) return n;
    return 1;
}

int log2_up(long v) { int b = 0; while (1l << b < v) ++b; return b; }
// vec: elements of a thread, as the rows' alignment allows (it moves the teams' borders, not a sum's order: that is given by the tiles, which come from the sizes)
Plan plan(int dt, long n, long C, int vec) {
    Plan p;
    const int most = dt ? 8 : 4;
    const long threads = (C + most - 1) / most;                 // of a tile, with whole vectors
    // Tiles: the shortest whose teams the device holds at once (three CTAs an SM), or, where even the longest are more, 32: many short waves instead of a little more than one.
    // 16384 x 1024 bf16 in tiles of 16, 32, 64, 128: 55, 49, 51, 68 us; 131072 x 1024: 205, 191, 193, 218; 131072 x 256: 69, 63, 59, 67; a million x 64: 275, 259, 236, 216.
    // At the border, 113664 x 1024 of 32000 rows, and behind it 32 is not the best: in tiles of 32, 64, 128 just under it 135, 128, 121 us (128 is taken), just over it 136, 126, 120 (32 is),
    // 250000 245, 233, 230; 131072 of 131072 rows 205, 202, 215.
    const long room = 148l * 3 * 256;
    int t = 16;
    while (t < 128 && (n + t - 1) / t * threads > room) t *= 2;
    if ((n + t - 1) / t * threads > room) t = 32;
    p.tile = t;
    p.tiles = (int)((n + t - 1) / t);
    p.tx = 1 << std::min(8, log2_up((C + vec - 1) / vec));
    p.slices = (int)(((C + vec - 1) / vec + p.tx - 1) / p.tx);
    return p;
}
// The workspace: two lists of the sort, and what the sums leave.
struct Space {
    size_t list, part, head, chain, bytes;
    Space(long n, long tiles, long C) {
        auto up = [](size_t v) { return (v + 255) / 256 * 256; };
        list = up((size_t)n * sizeof(uint2));
        part = 2 * list;
        head = part + up((size_t)tiles * C * sizeof(float));
        chain = head + up((size_t)tiles * sizeof(int));
        bytes = chain + up((size_t)(tiles + 1) * sizeof(int2));
    }
};

template <typename T>
cudaError_t forward_t(const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long ys, cudaStream_t s) {
    const int vec = std::min(vector<T>(table, C, C), vector<T>(y, ys, C));
    const unsigned per_row = (unsigned)(C / vec), row_step = 256 / per_row, col_step = 256 % per_row;
    const unsigned blocks = (unsigned)((n * per_row + 256 * UNROLL - 1) / (256 * UNROLL));
    auto go = [&](auto k) { return klaunch(k, blocks, 256, 0, s, tokens, (unsigned)n, (const T*)table, (unsigned)vocab, (int)C, per_row, row_step, col_step, scale, (T*)y, ys); };
    return vec == 1 ? go(embed_fwd_k<T, 1>) : vec == 2 ? go(embed_fwd_k<T, 2>) : go(embed_fwd_k<T, 16 / sizeof(T)>);
}

template <typename T, int N>
cudaError_t backward_t(int dt, const int32_t* tokens, long n, const T* dy, long dys, long vocab, long C, float scale, bool accum, float* dtable, char* ws, cudaStream_t s) {
    if (n <= FEW) {
        const int slices = (int)((C + 32 * N - 1) / (32 * N)), sum_ctas = (int)((n * slices + 7) / 8);
        const int fill_ctas = accum ? 0 : (int)std::min<long>(std::max<long>(1, vocab * C / 8192), 4 * 148);
        return klaunch(embed_few_k<T, N>, (unsigned)(sum_ctas + fill_ctas), 256, 0, s, tokens, (int)n, dy, dys, vocab, (int)C, slices, scale, (int)accum, dtable, sum_ctas);
    }
    const Plan p = plan(dt, n, C, N);
    const Space sp(n, p.tiles, C);
    uint2 *const list = (uint2*)ws, *const other = (uint2*)(ws + sp.list);
    unsigned* const counts = (unsigned*)(ws + sp.chain);
    const Left left{(float*)(ws + sp.part), (int*)(ws + sp.head), counts, counts + 1, (int2*)(counts + 2)};
    const int gs = log2_up((32 + C - 1) / C);                    // a group: 128 bytes of the table at least
    const long groups = ((vocab - 1) >> gs) + 1, rows = ((groups + OWNERS - 1) >> OWNER_BITS) << gs;      // rows of an owner, the last of which may be behind the table
    const int key_bits = log2_up(rows), passes = (key_bits + MAX_BITS - 1) / MAX_BITS, bits = passes ? (key_bits + passes - 1) / passes : 0;      // (none: an owner has one row)
    static OncePerDevice once;
    cudaError_t e = allow_smem(once, (const void*)embed_sort_k, SORT_WARPS * (1 << MAX_BITS) * (int)sizeof(unsigned));
    if (e != cudaSuccess) return e;
    e = klaunch(embed_sort_k, (unsigned)std::min<long>(groups, OWNERS), SORT_THREADS, (size_t)std::max(SORT_WARPS << bits, FILL_ROWS / 32) * sizeof(unsigned), s, tokens, (int)n, (unsigned)vocab,
                list, other, (int)rows, gs, passes, bits, accum ? nullptr : dtable, (int)C, (int)(N > 2), left.count, left.chains);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)((p.tiles + 256 / p.tx - 1) / (256 / p.tx)), (unsigned)p.slices);
    e = klaunch(embed_sums_k<T, N>, grid, 256, 0, s, (const uint2*)list, dy, dys, (int)C, scale, (int)accum, dtable, left, p);
    if (e != cudaSuccess) return e;
    constexpr int J = N > 2 ? 4 : 1;
    const dim3 joins((unsigned)std::min(p.tiles, 8 * 148), (unsigned)((C + J * JOIN_TX - 1) / (J * JOIN_TX)));
    return klaunch(embed_joins_k<J>, joins, 256, 0, s, (int)C, scale, dtable, left, p);
}

}  // namespace

cudaError_t embed_forward(int dt, const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long y_stride, cudaStream_t s) {
    if (n == 0) return cudaSuccess;
    Scope sc(KC_EMBED_FWD, (double)n * C, (double)n * (4 + 2.0 * C * (dt ? 2 : 4)), s);
    return dt ? forward_t<bf16>(tokens, n, table, vocab, C, scale, y, y_stride, s) : forward_t<float>(tokens, n, table, vocab, C, scale, y, y_stride, s);
}

size_t embed_workspace_bytes(long n, long, long C) {
    if (n <= FEW) return 0;
    return Space(n, std::max(plan(0, n, C, 1).tiles, plan(1, n, C, 1).tiles), C).bytes;
}

cudaError_t embed_backward(int dt, const int32_t* tokens, long n, const void* dy, long dy_stride, long vocab, long C, float scale, bool accum, float* dtable, void* ws,
                           cudaStream_t s) {
    if (n == 0 && accum) return cudaSuccess;
    Scope sc(KC_EMBED_GRAD, 2.0 * n * C, (double)n * (4 + C * (dt ? 2.0 : 4.0)) + (accum ? 0.0 : 4.0 * vocab * C), s);
    const bool rows = (uintptr_t)dtable % 16 == 0;              // whole vectors of dtable too
    auto go = [&](auto* p) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(p)>>;
        const int vec = vector<T>(p, dy_stride, C);
        if (vec > 2 && rows) return backward_t<T, 16 / sizeof(T)>(dt, tokens, n, p, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s);
        return vec > 1 ? backward_t<T, 2>(dt, tokens, n, p, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s)
                       : backward_t<T, 1>(dt, tokens, n, p, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s);
    };
    return dt ? go((const bf16*)dy) : go((const float*)dy);
}

}  // namespace fdg
