// Embedding lookup with scaling, y[i] = scale * table[tokens[i]], and the gradient of its table, dtable[v] = scale * sum of the dy rows whose token is v.
// Both move rows of C values and do next to nothing with them: the bound is HBM (lookup: rows read and written; gradient: dy read, the table's
// gradient written, zeros included).
//
// The gradient's sums are made in the order of the tokens' positions (in pieces of fixed size), never by atomic additions, so that equal inputs give equal bits.
// Few tokens: a warp per token looks through all of them.  Otherwise the positions are sorted by token (stable) and the sorted list is cut into tiles:
//   sort    one cluster of CTAs, a radix sort of 8 or 9 bits a pass through L2, while the other SMs fill the table's gradient with zeros
//   sums    a team of threads per tile adds the rows up, and writes a token's sum when the next one begins; a sum that began in an earlier tile is left as
//           a partial row
//   joins   the team of the tile in which a token began adds the partial rows of the following tiles to its row
#include "seqops.h"
#include "launch.h"

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

namespace fdg {
namespace {

namespace cg = cooperative_groups;
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

// ---- lookup: every thread moves UNROLL vectors of the output, neighbours side by side
constexpr int UNROLL = 4;
template <typename T, int N>
__global__ void __launch_bounds__(256) embed_fwd_k(const int32_t* __restrict__ tokens, long n, const T* __restrict__ table, unsigned vocab, int C, int per_row, float scale,
                                                   T* __restrict__ y, long ys) {
    const long begin = (long)blockIdx.x * (256 * UNROLL), row0 = begin / per_row;
    const unsigned rest = (unsigned)(begin - row0 * per_row);
    Raw<T, N> r[UNROLL];
    long row[UNROLL];
    unsigned col[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const unsigned at = rest + u * 256 + threadIdx.x, k = at / (unsigned)per_row;
        row[u] = row0 + k; col[u] = (at - k * per_row) * N;
        r[u] = Raw<T, N>{};
        if (row[u] < n) {
            const unsigned tok = (unsigned)tokens[row[u]];               // negative ids are large ones
            if (tok < vocab) r[u] = *(const Raw<T, N>*)(table + (long)tok * C + col[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        if (row[u] >= n) continue;
        float x[N];
        unpack<T, N>(r[u], x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= scale;
        *(Raw<T, N>*)(y + row[u] * ys + col[u]) = pack<T, N>(x);
    }
}

// ---- gradient of few tokens, in one launch
constexpr long FEW = 512;
constexpr int FILL_ROWS = 4096;                 // rows of the table that a filling CTA looks at a time
// zeros to elements [lo, hi) of p by the CTA; p on 4 bytes
__device__ __forceinline__ void zero(float* p, long lo, long hi) {
    const long a = min(hi, lo + (long)((16 - (uintptr_t)(p + lo) % 16) % 16 / 4)), b = a + (hi - a) / 4 * 4;
    for (long i = lo + threadIdx.x; i < a; i += blockDim.x) p[i] = 0.f;
    for (long i = a + 4 * (long)threadIdx.x; i < b; i += 4 * (long)blockDim.x) *(float4*)(p + i) = make_float4(0.f, 0.f, 0.f, 0.f);
    for (long i = b + threadIdx.x; i < hi; i += blockDim.x) p[i] = 0.f;
}
// CTAs 0 .. warps / 8 - 1: a warp per token and 32 N channels; it goes on if no earlier token is the same, and adds up all that are, in order.  The
// others fill the rows that no token names.
template <typename T, int N>
__global__ void __launch_bounds__(256) embed_few_k(const int32_t* __restrict__ tokens, int n, const T* __restrict__ dy, long dys, long vocab, int C, int slices, float scale,
                                                   int accum, float* __restrict__ dtable, int sum_ctas) {
    if ((int)blockIdx.x >= sum_ctas) {
        __shared__ unsigned named[FILL_ROWS / 32];
        const long ctas = gridDim.x - sum_ctas, per = (vocab + ctas - 1) / ctas, r0 = (blockIdx.x - sum_ctas) * per, r1 = min(vocab, r0 + per);
        for (long b = r0; b < r1; b += FILL_ROWS) {
            const int rows = (int)min((long)FILL_ROWS, r1 - b);
            __syncthreads();
            for (int i = threadIdx.x; i < FILL_ROWS / 32; i += 256) named[i] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += 256) { const long t = tokens[i] - b; if (t >= 0 && t < rows) atomicOr(&named[t >> 5], 1u << (t & 31)); }
            __syncthreads();
            for (int r = 0; r < rows;) {                        // runs of rows without a token
                int e = r;
                while (e < rows && !(named[e >> 5] >> (e & 31) & 1)) e = named[e >> 5] == 0 && (e & 31) == 0 ? min(rows, e + 32) : e + 1;
                if (e > r) zero(dtable, (b + r) * C, (b + e) * C);
                r = e + 1;
            }
        }
        return;
    }
    const int warp = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, i = warp / slices, c = (warp - i * slices) * 32 * N + lane * N;
    if (i >= n) return;
    const int tok = tokens[i];
    if (tok < 0 || tok >= vocab) return;
    for (int j = 0; j < i; j += 128) {
        bool same = false;
#pragma unroll
        for (int u = 0; u < 4; ++u) { const int q = j + u * 32 + lane; same |= q < i && tokens[q] == tok; }
        if (__any_sync(~0u, same)) return;
    }
    const bool in = c < C;
    float sum[N] = {};
    for (int j = i; j < n; j += 32) {
        unsigned hits = __ballot_sync(~0u, j + lane < n && tokens[j + lane] == tok);
        while (hits) {
            Raw<T, N> r[4];
            int m = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (hits) { const int q = __ffs(hits) - 1; hits &= hits - 1; m = u + 1; if (in) r[u] = *(const Raw<T, N>*)(dy + (j + q) * dys + c); }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u < m && in) {
                    float x[N];
                    unpack<T, N>(r[u], x);
#pragma unroll
                    for (int k = 0; k < N; ++k) sum[k] += x[k];
                }
        }
    }
    if (!in) return;
    float* const d = dtable + (long)tok * C + c;
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] = accum ? fmaf(sum[k], scale, d[k]) : sum[k] * scale;
}

// ---- gradient of many tokens
constexpr int SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32, MAX_BITS = 9, MAX_CLUSTER = 8, AHEAD = 8;

// entries of the sorted list: token (ids outside the table: vocab, so that they come last) and position
__global__ void __launch_bounds__(SORT_THREADS) embed_sort_k(const int32_t* __restrict__ tokens, int n, unsigned vocab, uint2* buf0, uint2* buf1, int passes, int bits, int S,
                                                             float* dtable, long fill) {
    if (blockIdx.x >= S) {                                      // not the sorting cluster
        const long ctas = gridDim.x - S, per = ((fill + ctas - 1) / ctas + 3) / 4 * 4, lo = min(fill, (blockIdx.x - S) * per);
        zero(dtable, lo, min(fill, lo + per));
        return;
    }
    extern __shared__ unsigned hist[];                          // [warp][bin]
    __shared__ unsigned total[1 << MAX_BITS], base[1 << MAX_BITS], sums[SORT_WARPS];
    cg::cluster_group cl = cg::this_cluster();
    const int rank = blockIdx.x, w = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << bits;
    const int per_warp = ((n + S * SORT_WARPS - 1) / (S * SORT_WARPS) + 31) / 32 * 32;
    const long b0 = (long)(rank * SORT_WARPS + w) * per_warp;
    const int begin = (int)min((long)n, b0), end = (int)min((long)n, b0 + per_warp);
    unsigned* const mine = hist + w * bins;
    for (int p = 0; p < passes; ++p) {
        const int shift = p * bits;
        const uint2* const src = p & 1 ? buf0 : buf1;
        uint2* const dst = p & 1 ? buf1 : buf0;
        // entries begin + 32 k + lane of the warp, k by k, to f(entry, its digit (or `bins` behind the end), lanes of equal digit)
        auto each = [&](auto f) {
            for (int i0 = begin; i0 < end; i0 += 32 * AHEAD) {
                uint2 e[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int i = i0 + u * 32 + lane;
                    if (i >= end) continue;
                    if (p == 0) { const unsigned t = (unsigned)tokens[i]; e[u] = make_uint2(t < vocab ? t : vocab, (unsigned)i); }
                    else e[u] = __ldcg(src + i);
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (i0 + u * 32 >= end) break;
                    const unsigned d = i0 + u * 32 + lane < end ? e[u].x >> shift & (bins - 1) : (unsigned)bins;
                    f(e[u], d, __match_any_sync(~0u, d));
                }
            }
        };
        for (int i = threadIdx.x; i < SORT_WARPS * bins; i += SORT_THREADS) hist[i] = 0;
        __syncthreads();
        each([&](const uint2&, unsigned d, unsigned peers) {
            if (d < bins && lane == __ffs(peers) - 1) mine[d] += __popc(peers);
            __syncwarp();
        });
        __syncthreads();
        // of every bin: its entries in the warps in front, in the CTA
        for (int b = threadIdx.x; b < bins; b += SORT_THREADS) {
            unsigned run = 0;
#pragma unroll 8
            for (int q = 0; q < SORT_WARPS; ++q) { const unsigned t = hist[q * bins + b]; hist[q * bins + b] = run; run += t; }
            total[b] = run;
        }
        cl.sync();
        // where the CTA's part of every bin begins: behind all smaller bins and the CTAs in front
        unsigned all = 0, front = 0;
        const int b = threadIdx.x;
        if (b < bins)
            for (int r = 0; r < S; ++r) { const unsigned t = *cl.map_shared_rank(&total[b], r); all += t; if (r < rank) front += t; }
        unsigned scan = all;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) { const unsigned t = __shfl_up_sync(~0u, scan, d); if (lane >= d) scan += t; }
        if (lane == 31) sums[w] = scan;
        __syncthreads();
        if (b < bins) {
            unsigned before = scan - all + front;
            for (int q = 0; q < w; ++q) before += sums[q];
            base[b] = before;
        }
        __syncthreads();
        each([&](const uint2& e, unsigned d, unsigned peers) {
            const unsigned at = d < bins ? mine[d] : 0;
            __syncwarp();
            if (d < bins) {
                if (lane == __ffs(peers) - 1) mine[d] = at + __popc(peers);
                dst[base[d] + at + __popc(peers & ((1u << lane) - 1))] = e;
            }
            __syncwarp();
        });
        cl.sync();                                              // the list is whole, and nobody reads `total` any more
    }
}

// How the sorted list is cut: tiles of `tile` entries, each summed by teams of `tx` threads (of which `slices` cover the channels).
struct Plan { int vec, tx, slices, tile; long tiles; };

constexpr int BATCH = 8;                        // rows on their way at once
template <typename T, int N>
__global__ void __launch_bounds__(256) embed_sums_k(const uint2* __restrict__ list, int n, const T* __restrict__ dy, long dys, unsigned vocab, int C, float scale, int accum,
                                                    float* __restrict__ dtable, float* __restrict__ part, Plan p) {
    const long tile = (long)blockIdx.x * (256 / p.tx) + threadIdx.x / p.tx;
    const int c = (blockIdx.y * p.tx + threadIdx.x % p.tx) * N;
    if (tile >= p.tiles || c >= C) return;
    const int t0 = (int)(tile * p.tile), t1 = min(n, t0 + p.tile);
    unsigned now = list[t0].x;
    bool begun = t0 > 0 && list[t0 - 1].x == now;               // in an earlier tile
    float sum[N] = {};
    auto leave = [&]() {
        if (now >= vocab) return;
        float* const d = begun ? part + tile * C + c : dtable + (long)now * C + c;
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
            const uint2 e = i + u < t1 ? list[i + u] : make_uint2(vocab, 0);
            key[u] = e.x;
            if (e.x < vocab) r[u] = *(const Raw<T, N>*)(dy + (long)e.y * dys + c);
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
            if (now < vocab) {
                float x[N];
                unpack<T, N>(r[u], x);
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] += x[k];
            }
        }
    }
    leave();
}

// Here a thread has 4 channels (N = 4, rows on 16 bytes) or one; tx of them make a team.
constexpr int JOIN_BATCH = 16;
template <int N>
__global__ void __launch_bounds__(256) embed_joins_k(const uint2* __restrict__ list, int n, unsigned vocab, int C, float scale, float* __restrict__ dtable,
                                                     const float* __restrict__ part, long tiles, int tile_, int tx) {
    const long tile = (long)blockIdx.x * (256 / tx) + threadIdx.x / tx;
    const int c = (blockIdx.y * tx + threadIdx.x % tx) * N;
    if (tile + 1 >= tiles || c >= C) return;
    const long t0 = tile * tile_, t1 = t0 + tile_;
    const unsigned now = list[t1 - 1].x;
    if (now >= vocab || list[t1].x != now) return;              // nothing goes on behind this tile
    if (t0 > 0 && list[t0].x == now && list[t0 - 1].x == now) return;        // it began before this tile
    float sum[N] = {};
    for (long j = tile + 1; j < tiles; j += JOIN_BATCH) {
        bool more[JOIN_BATCH];
        Raw<float, N> v[JOIN_BATCH];
#pragma unroll
        for (int u = 0; u < JOIN_BATCH; ++u) {
            more[u] = j + u < tiles && list[(j + u) * tile_].x == now;
            if (more[u]) v[u] = *(const Raw<float, N>*)(part + (j + u) * C + c);
        }
#pragma unroll
        for (int u = 0; u < JOIN_BATCH; ++u)
            if (more[u]) {
                float x[N];
                unpack<float, N>(v[u], x);
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] += x[k];
            }
        if (!more[JOIN_BATCH - 1]) break;
    }
    float* const d = dtable + (long)now * C + c;
#pragma unroll
    for (int k = 0; k < N; ++k) d[k] = fmaf(sum[k], scale, d[k]);
}

// elements that may be moved at once
template <typename T> int vector(const void* a, long stride_a, long C) {
    for (int n = 16 / (int)sizeof(T); n > 1; n = 1) if ((uintptr_t)a % 16 == 0 && stride_a % n == 0 && C % n == 0) return n;
    return 1;
}

int log2_up(long v) { int b = 0; while (1l << b < v) ++b; return b; }
// vec: as the rows' alignment allows (it moves the teams' borders, not a sum's order: that is given by the tiles, which come from the sizes)
Plan plan(int dt, long n, long C, int vec) {
    Plan p;
    const int most = dt ? 8 : 4;
    const long threads = (C + most - 1) / most;                 // of a tile, with whole vectors
    // tiles: enough teams for a quarter of the device's threads, of 16 to 128 entries (longer ones leave fewer partial rows to join, and fewer teams)
    int t = 16;
    while (t < 128 && (n / (2 * t)) * threads >= 148l * 512) t *= 2;
    p.tile = t;
    p.tiles = (n + t - 1) / t;
    p.vec = vec;
    p.tx = 1 << std::min(8, log2_up((C + vec - 1) / vec));
    p.slices = (int)(((C + vec - 1) / vec + p.tx - 1) / p.tx);
    return p;
}

template <typename T>
cudaError_t forward_t(const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long ys, cudaStream_t s) {
    const int vec = std::min(vector<T>(table, C, C), vector<T>(y, ys, C));
    const int per_row = (int)(C / vec);
    const unsigned blocks = (unsigned)((n * per_row + 256 * UNROLL - 1) / (256 * UNROLL));
    if (vec == 1) return klaunch(embed_fwd_k<T, 1>, blocks, 256, 0, s, tokens, n, (const T*)table, (unsigned)vocab, (int)C, per_row, scale, (T*)y, ys);
    return klaunch(embed_fwd_k<T, 16 / sizeof(T)>, blocks, 256, 0, s, tokens, n, (const T*)table, (unsigned)vocab, (int)C, per_row, scale, (T*)y, ys);
}

template <typename T, int N>
cudaError_t backward_t(int dt, const int32_t* tokens, long n, const T* dy, long dys, long vocab, long C, float scale, bool accum, float* dtable, char* ws, cudaStream_t s) {
    if (n <= FEW) {
        const int slices = (int)((C + 32 * N - 1) / (32 * N)), sum_ctas = (int)((n * slices + 7) / 8);
        const int fill_ctas = accum ? 0 : (int)std::min<long>(std::max<long>(1, vocab * C / 8192), 4 * 148);
        return klaunch(embed_few_k<T, N>, (unsigned)(sum_ctas + fill_ctas), 256, 0, s, tokens, (int)n, dy, dys, vocab, (int)C, slices, scale, (int)accum, dtable, sum_ctas);
    }
    const Plan p = plan(dt, n, C, N);
    const size_t list_bytes = ((size_t)n * sizeof(uint2) + 255) / 256 * 256;
    uint2 *const buf0 = (uint2*)ws, *const buf1 = (uint2*)(ws + list_bytes);
    float* const part = (float*)(ws + 2 * list_bytes);
    const int key_bits = log2_up(vocab + 1), passes = (key_bits + MAX_BITS - 1) / MAX_BITS, bits = (key_bits + passes - 1) / passes;
    int S = 1;
    while (S < MAX_CLUSTER && n > 2048l * S) S *= 2;
    const long fill = accum ? 0 : vocab * C;
    const int fill_ctas = (int)(std::min<long>((fill + 65535) / 65536, 2 * 148) + S - 1) / S * S;
    const size_t smem = (size_t)SORT_WARPS * (1 << bits) * sizeof(unsigned);
    static OncePerDevice once;
    cudaError_t e = allow_smem(once, (const void*)embed_sort_k, SORT_WARPS * (1 << MAX_BITS) * sizeof(unsigned));
    if (e != cudaSuccess) return e;
    e = klaunch_cluster(embed_sort_k, (unsigned)(S + fill_ctas), SORT_THREADS, smem, s, S, tokens, (int)n, (unsigned)vocab, buf0, buf1, passes, bits, S, dtable, fill);
    if (e != cudaSuccess) return e;
    const uint2* const list = passes & 1 ? buf0 : buf1;
    const dim3 grid((unsigned)((p.tiles + 256 / p.tx - 1) / (256 / p.tx)), (unsigned)p.slices);
    e = klaunch(embed_sums_k<T, N>, grid, 256, 0, s, list, (int)n, dy, dys, (unsigned)vocab, (int)C, scale, (int)accum, dtable, part, p);
    if (e != cudaSuccess || p.tiles == 1) return e;
    const int jv = N > 1 ? 4 : 1, tx = 1 << std::min(8, log2_up((C + jv - 1) / jv));
    const dim3 jgrid((unsigned)((p.tiles + 256 / tx - 1) / (256 / tx)), (unsigned)((C + (long)jv * tx - 1) / ((long)jv * tx)));
    return klaunch(embed_joins_k<(N > 1 ? 4 : 1)>, jgrid, 256, 0, s, list, (int)n, (unsigned)vocab, (int)C, scale, dtable, (const float*)part, p.tiles, p.tile, tx);
}

}  // namespace

cudaError_t embed_forward(int dt, const int32_t* tokens, long n, const void* table, long vocab, long C, float scale, void* y, long y_stride, cudaStream_t s) {
    if (n == 0) return cudaSuccess;
    Scope sc(KC_EMBED_FWD, (double)n * C, (double)n * (4 + 2.0 * C * (dt ? 2 : 4)), s);
    return dt ? forward_t<bf16>(tokens, n, table, vocab, C, scale, y, y_stride, s) : forward_t<float>(tokens, n, table, vocab, C, scale, y, y_stride, s);
}

size_t embed_workspace_bytes(long n, long, long C) {
    if (n <= FEW) return 0;
    const long tiles = std::max(plan(0, n, C, 1).tiles, plan(1, n, C, 1).tiles);
    return 2 * (((size_t)n * sizeof(uint2) + 255) / 256 * 256) + (size_t)tiles * C * sizeof(float);
}

cudaError_t embed_backward(int dt, const int32_t* tokens, long n, const void* dy, long dy_stride, long vocab, long C, float scale, bool accum, float* dtable, void* ws,
                           cudaStream_t s) {
    if (n == 0 && accum) return cudaSuccess;
    Scope sc(KC_EMBED_GRAD, 2.0 * n * C, (double)n * (4 + C * (dt ? 2.0 : 4.0)) + (accum ? 0.0 : 4.0 * vocab * C), s);
    const bool rows = (uintptr_t)dtable % 16 == 0;              // whole vectors of dtable too
    if (dt) return rows && vector<bf16>(dy, dy_stride, C) > 1 ? backward_t<bf16, 8>(dt, tokens, n, (const bf16*)dy, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s)
                                                             : backward_t<bf16, 1>(dt, tokens, n, (const bf16*)dy, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s);
    return rows && vector<float>(dy, dy_stride, C) > 1 ? backward_t<float, 4>(dt, tokens, n, (const float*)dy, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s)
                                                       : backward_t<float, 1>(dt, tokens, n, (const float*)dy, dy_stride, vocab, C, scale, accum, dtable, (char*)ws, s);
}

}  // namespace fdg
