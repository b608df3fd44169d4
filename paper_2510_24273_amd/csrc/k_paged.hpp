// Paged full-rank key-value cache: append of new tokens, attention of one new token per sequence, eviction of tokens by
// accumulated attention weight.
//
// Slot j of sequence b is row j % page_size of page table[b, j / page_size]; a row holds [H_kv, D] elements, K already rotated.
#pragma once
#include "common.hpp"

namespace sals {

constexpr double kInvTwoPi = 0.15915494309189533576888376337251;

// n / d for 0 <= n <= 2^20 and 1 <= d <= 2048 by one multiplication: with m = ceil(2^31 / d) = (2^31 + e) / d, e < d, the quotient
// 2n m / 2^32 = n / d + n e / (2^31 d) stays below the next whole number as long as n e < 2^31.
__device__ __forceinline__ uint32_t page_of(uint32_t n, uint32_t m) { return __umulhi(2u * n, m); }

struct PagedCache {           // the cache of one layer and the shape of the call
    const int32_t* table;     // [B, max_pages]
    const int32_t* seq_len;   // [B]
    int64_t page_stride;      // elements
    uint32_t page_mul;        // ceil(2^31 / page_size)
    int32_t page_size, max_pages, n_pages, cap;   // cap = max_pages * page_size
    int32_t B, H_kv, group;   // group: query heads of a KV head
};

// cos / sin of position * theta^(-2 pair / D): the angle in turns, in fp64, less its whole part; what is left is exact to 1e-16 * position
// turns and goes to fp32 (half a step of a value of at most 1/2 turn: 9e-8 radians).
template <int D> __device__ __forceinline__ float2 rope_turn(int position, int pair, double log2_theta)
{
    const double t = (double)position * (exp2(-(double)pair * (2.0 / D) * log2_theta) * kInvTwoPi);
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    return make_float2(c, s);
}
template <int D> __device__ __forceinline__ int pair_lo(int p, int style) { return style ? 2 * p : p; }
template <int D> __device__ __forceinline__ int pair_hi(int p, int style) { return style ? 2 * p + 1 : p + D / 2; }

// element offset of slot j's row, or -1 where its page is not there
__device__ __forceinline__ int64_t paged_row(const PagedCache& a, int b, int j, int row)
{
    const uint32_t pg = page_of((uint32_t)j, a.page_mul);
    const int32_t id = a.table[(size_t)b * a.max_pages + pg];
    return (uint32_t)id < (uint32_t)a.n_pages ? (int64_t)id * a.page_stride + (int64_t)(j - (int)pg * a.page_size) * row : -1;
}

// ---- append ---------------------------------------------------------------------------------------------------------------------
// A workgroup takes kAppTok consecutive new tokens of a sequence, all heads: cos / sin of its tokens once into LDS, then 16-byte
// pieces.  With one workgroup per sequence (n_tok <= kAppTok) it advances the length itself, behind its own reading of it.
constexpr int kAppTok = 8;

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedCache a, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                           const int32_t* __restrict__ q_pos, T* __restrict__ Kp, T* __restrict__ Vp,
                                                           int32_t* seq_len, const int32_t* __restrict__ n_new, int n_tok,
                                                           int32_t* __restrict__ pos, float* __restrict__ weights, int lists,
                                                           double log2_theta, int style)
{
    constexpr int VEC = elem<T>::vec, NP = D / 2, PIECES = D / VEC;
    __shared__ float2 sCS[kAppTok][NP];
    __shared__ int64_t sRow[kAppTok];
    const int b = blockIdx.y, t0 = blockIdx.x * kAppTok, tid = threadIdx.x;
    const int have = min(max(seq_len[b], 0), a.cap);
    const int want = n_new ? min(max(n_new[b], 0), n_tok) : n_tok;
    const int n = min(want, a.cap - have);          // tokens that fit
    const int nt = min(kAppTok, n - t0);
    const int row = a.H_kv * D, qp = q_pos[b];
    for (int i = tid; i < nt * NP; i += 256) sCS[i / NP][i % NP] = rope_turn<D>(qp + t0 + i / NP, i % NP, log2_theta);
    if (tid < nt) sRow[tid] = paged_row(a, b, have + t0 + tid, row);
    __syncthreads();
    if (gridDim.x == 1 && tid == 0 && n > 0) seq_len[b] = have + n;
    for (int i = tid; i < nt * lists; i += 256) {
        const size_t at = ((size_t)b * lists + i / nt) * a.cap + have + t0 + i % nt;
        pos[at] = qp + t0 + i % nt;
        weights[at] = 0.f;
    }
    const int pieces = a.H_kv * PIECES;              // of a token
    for (int i = tid; i < nt * pieces; i += 256) {
        const int t = i / pieces, pc = i - t * pieces;
        const int64_t at = sRow[t];
        if (at < 0) continue;
        const size_t from = ((size_t)b * n_tok + t0 + t) * row + (size_t)pc * VEC;
        *reinterpret_cast<u32x4*>(Vp + at + (size_t)pc * VEC) = ld16(v_new + from);
        // a piece of K and the piece of its partners: the same one for neighbouring pairs, half a head away otherwise
        const int ch = pc % PIECES * VEC;
        float x[VEC], y[VEC], r[VEC];
        elem<T>::unpack(ld16(k_new + from), x);
        if (style) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const float2 cs = sCS[t][(ch + e) / 2];
                r[e] = fmaf(x[e], cs.x, -(x[e + 1] * cs.y));
                r[e + 1] = fmaf(x[e + 1], cs.x, x[e] * cs.y);
            }
        } else {
            const bool first = ch < NP;
            elem<T>::unpack(ld16(k_new + (first ? from + NP : from - NP)), y);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float2 cs = sCS[t][(ch + e) % NP];
                r[e] = fmaf(x[e], cs.x, first ? -(y[e] * cs.y) : y[e] * cs.y);
            }
        }
        u32x4 w;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (uint32_t)f32_to_bf16(r[2 * e]) | (uint32_t)f32_to_bf16(r[2 * e + 1]) << 16;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(r[e]);
        }
        *reinterpret_cast<u32x4*>(Kp + at + (size_t)pc * VEC) = w;
    }
}

// the lengths behind an append of several workgroups per sequence
__global__ __launch_bounds__(256) void paged_advance_kernel(int32_t* seq_len, const int32_t* __restrict__ n_new, int n_tok, int cap, int B)
{
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= B) return;
    const int have = min(max(seq_len[b], 0), cap), want = n_new ? min(max(n_new[b], 0), n_tok) : n_tok;
    const int n = min(want, cap - have);
    if (n > 0) seq_len[b] = have + n;
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
// Logits are kept in units of ln 2 (the query is scaled by log2(e) / sqrt(D)), so that exponentials are powers of two.
constexpr int kPgHeads = 16;           // query heads of a workgroup

// grid (chunks, H_kv * head tiles, B): a wave takes a token at a time, a lane D / 64 channels of it
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_attend_kernel(PagedCache a, const T* __restrict__ q, const int32_t* __restrict__ q_pos,
                                                           const T* __restrict__ Kp, const T* __restrict__ Vp, float* __restrict__ part,
                                                           float* __restrict__ logits, float scale, double log2_theta, int style)
{
    constexpr int CPL = D / 64, REC = D + 2;
    __shared__ float sQ[kPgHeads][D];
    __shared__ float2 sCS[D / 2];
    __shared__ float sRed[4][REC];
    const int chunk = blockIdx.x, n_chunks = gridDim.x, b = blockIdx.z;
    const int tiles = (a.group + kPgHeads - 1) / kPgHeads, g = blockIdx.y / tiles, h0 = blockIdx.y % tiles * kPgHeads;
    const int nh = min(kPgHeads, a.group - h0), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = a.H_kv * a.group;
    const int S = min(max(a.seq_len[b], 0), a.cap);
    const int per = ((S + n_chunks - 1) / n_chunks + 3) & ~3, j0 = min(S, chunk * per), j1 = min(S, j0 + per);
    if (tid < D / 2) sCS[tid] = rope_turn<D>(q_pos[b], tid, log2_theta);
    __syncthreads();
    for (int i = tid; i < nh * (D / 2); i += 256) {
        const int m = i / (D / 2), p = i % (D / 2), c1 = pair_lo<D>(p, style), c2 = pair_hi<D>(p, style);
        const T* qh = q + ((size_t)b * H + (size_t)g * a.group + h0 + m) * D;
        const float x = elem<T>::load(qh + c1), y = elem<T>::load(qh + c2);
        sQ[m][c1] = (x * sCS[p].x - y * sCS[p].y) * scale;
        sQ[m][c2] = (y * sCS[p].x + x * sCS[p].y) * scale;
    }
    __syncthreads();
    float mx[kPgHeads], l[kPgHeads], acc[kPgHeads][CPL];
#pragma unroll
    for (int m = 0; m < kPgHeads; ++m) {
        mx[m] = -INFINITY; l[m] = 0.f;
        for (int c = 0; c < CPL; ++c) acc[m][c] = 0.f;
    }
    const int row = a.H_kv * D;
    for (int j = j0 + wave; j < j1; j += 4) {
        const int64_t at = paged_row(a, b, j, row);
        float k[CPL], v[CPL];
        if (at >= 0)
            for (int c = 0; c < CPL; ++c) {
                k[c] = elem<T>::load(Kp + at + g * D + lane * CPL + c);
                v[c] = elem<T>::load(Vp + at + g * D + lane * CPL + c);
            }
#pragma unroll
        for (int m = 0; m < kPgHeads; ++m) {
            if (m >= nh) continue;
            float x = -INFINITY;
            if (at >= 0) {
                x = 0.f;
                for (int c = 0; c < CPL; ++c) x = fmaf(sQ[m][lane * CPL + c], k[c], x);
                x = wave_sum(x);
                const float mn = fmaxf(mx[m], x), r = exp2f(mx[m] - mn), p = exp2f(x - mn);
                mx[m] = mn;
                l[m] = l[m] * r + p;
                for (int c = 0; c < CPL; ++c) acc[m][c] = fmaf(p, v[c], acc[m][c] * r);
            }
            if (logits && lane == 0) logits[((size_t)b * H + (size_t)g * a.group + h0 + m) * a.cap + j] = x;
        }
    }
    for (int m = 0; m < kPgHeads; ++m) {
        if (m >= nh) break;
        __syncthreads();
        if (lane == 0) { sRed[wave][0] = mx[m]; sRed[wave][1] = l[m]; }
        for (int c = 0; c < CPL; ++c) sRed[wave][2 + lane * CPL + c] = acc[m][c];
        __syncthreads();
        if (tid < D) {
            float M = -INFINITY, L = 0.f, A = 0.f;
            for (int w = 0; w < 4; ++w) M = fmaxf(M, sRed[w][0]);
            for (int w = 0; w < 4 && M > -INFINITY; ++w) {
                const float f = exp2f(sRed[w][0] - M);
                L = fmaf(sRed[w][1], f, L);
                A = fmaf(sRed[w][2 + tid], f, A);
            }
            float* rec = part + (((size_t)b * H + (size_t)g * a.group + h0 + m) * n_chunks + chunk) * REC;
            if (tid == 0) { rec[0] = M; rec[1] = L; }
            rec[2 + tid] = A;
        }
    }
}

// grid (B * H): the chunks joined; (maximum, 1 / sum) left for the weights
template <typename T, int D>
__global__ __launch_bounds__(D) void paged_merge_kernel(const float* __restrict__ part, T* __restrict__ out, float2* __restrict__ stat, int n_chunks)
{
    const size_t bh = blockIdx.x;
    const float* rec = part + bh * n_chunks * (D + 2);
    float M = -INFINITY, L = 0.f, A = 0.f;
    for (int k = 0; k < n_chunks; ++k) M = fmaxf(M, rec[(size_t)k * (D + 2)]);
    for (int k = 0; k < n_chunks && M > -INFINITY; ++k) {
        const float* r = rec + (size_t)k * (D + 2);
        const float f = exp2f(r[0] - M);
        L = fmaf(r[1], f, L);
        A = fmaf(r[2 + threadIdx.x], f, A);
    }
    elem<T>::store(out + bh * D + threadIdx.x, L > 0.f ? A / L : 0.f);
    if (threadIdx.x == 0) stat[bh] = make_float2(L > 0.f ? M : 0.f, L > 0.f ? 1.f / L : 0.f);
}

// weights[b, list, j] += sum over the list's heads of the softmax weight.  grid (x, lists, B)
__global__ __launch_bounds__(256) void paged_weights_kernel(PagedCache a, const float* __restrict__ logits, const float2* __restrict__ stat,
                                                            float* __restrict__ weights)
{
    const int lists = gridDim.y, b = blockIdx.z, H = a.H_kv * a.group, nh = H / lists, h0 = blockIdx.y * nh;
    const int S = min(max(a.seq_len[b], 0), a.cap);
    float* w = weights + ((size_t)b * lists + blockIdx.y) * a.cap;
    for (int j = blockIdx.x * 256 + threadIdx.x; j < S; j += gridDim.x * 256) {
        float sum = 0.f;
        for (int h = 0; h < nh; ++h) {
            const float2 st = stat[(size_t)b * H + h0 + h];
            sum += exp2f(logits[((size_t)b * H + h0 + h) * a.cap + j] - st.x) * st.y;
        }
        w[j] += sum;
    }
}

// ---- eviction -------------------------------------------------------------------------------------------------------------------
constexpr int kEvThreads = 1024;
constexpr int kEvBins = 2048;

struct EvictArgs {
    const int32_t* q_pos;
    int32_t* pos;
    float* weights;
    int32_t *src, *moves, *from, *to;   // moves [rows]: rows to move, -1 for none and no change of the length; from, to [rows, move_cap]
    int lists, n_keep, n_sink, n_recent, move_cap;
};

// what a slot is ranked by: NaN below all weights, protected ones above all
__device__ __forceinline__ uint32_t evict_key(float w, int32_t p, int32_t n_sink, int64_t recent_from)
{
    return p < n_sink || (int64_t)p > recent_from ? 0xffffffffu : w != w ? 0u : score_key(w);
}

// exclusive prefix sum over the workgroup's 16 waves; a barrier inside, another one before the next call's
__device__ __forceinline__ uint32_t evict_scan(uint32_t v, uint32_t* sums, uint32_t* total)
{
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const uint32_t iv = wave_incl_scan(v);
    __syncthreads();
    if (lane == kWave - 1) sums[wave] = iv;
    __syncthreads();
    const uint32_t w = sums[lane & 15];
    *total = row16_sum_u32(w);
    return row16_sum_u32((lane & 15) < wave ? w : 0u) + iv - v;
}

// One workgroup per list: radix select over the 32-bit keys (11 + 11 + 10 bits) for the key of the n_keep-th slot, then the slots
// in order: which stay, which become free below n_keep, which move.
__global__ __launch_bounds__(kEvThreads) void paged_evict_select_kernel(PagedCache a, EvictArgs e)
{
    __shared__ uint32_t hist[kEvBins];
    __shared__ uint32_t sums[16];
    __shared__ uint32_t sPrefix, sNeed;
    const int rowi = blockIdx.x, b = rowi / e.lists, tid = threadIdx.x;
    const int S = min(max(a.seq_len[b], 0), a.cap);
    int32_t* src = e.src ? e.src + (size_t)rowi * e.n_keep : nullptr;
    if (S <= e.n_keep) {
        if (src)
            for (int j = tid; j < e.n_keep; j += kEvThreads) src[j] = j < S ? j : -1;
        if (tid == 0) e.moves[rowi] = -1;
        return;
    }
    const float* w = e.weights + (size_t)rowi * a.cap;
    const int32_t* p = e.pos + (size_t)rowi * a.cap;
    const int64_t recent_from = (int64_t)e.q_pos[b] - e.n_recent;
    auto key_of = [&](int j) { return evict_key(w[j], p[j], e.n_sink, recent_from); };
    uint32_t prefix = 0, need = (uint32_t)e.n_keep;   // of the slots whose leading bits equal the prefix, `need` stay
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        for (int i = tid; i < kEvBins; i += kEvThreads) hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < S; j += kEvThreads) {
            const uint32_t k = key_of(j);
            if (pass == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[k >> shift & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // thread t holds bins kEvBins-1-2t and the one below: sums from the top
        const uint32_t c0 = hist[kEvBins - 1 - 2 * tid], c1 = hist[kEvBins - 2 - 2 * tid];
        uint32_t total;
        const uint32_t above = evict_scan(c0 + c1, sums, &total);
        if (above < need && need <= above + c0 + c1) {
            const bool second = need > above + c0;
            sPrefix = prefix << bits | (uint32_t)(kEvBins - 1 - 2 * tid - (second ? 1 : 0));
            sNeed = need - above - (second ? c0 : 0);
        }
        __syncthreads();
        prefix = sPrefix;
        need = sNeed;
    }
    uint32_t ties = 0, n_free = 0, n_late = 0;
    for (int base = 0; base < S; base += 4 * kEvThreads) {
        uint32_t key[4];
        uint32_t eq = 0;
        for (int u = 0; u < 4; ++u) {
            const int j = base + 4 * tid + u;
            key[u] = j < S ? key_of(j) : 0u;
            eq += j < S && key[u] == prefix;
        }
        uint32_t total;
        uint32_t rank = ties + evict_scan(eq, sums, &total);
        ties += total;
        uint32_t mine = 0;   // free slots, and moving ones in the upper half
        int what[4];
        for (int u = 0; u < 4; ++u) {
            const int j = base + 4 * tid + u;
            const bool tie = j < S && key[u] == prefix;
            const bool kept = j < S && (key[u] > prefix || (tie && rank < need));
            rank += tie;
            what[u] = j >= S || kept == (j < e.n_keep) ? 0 : kept ? 2 : 1;
            mine += what[u] == 1 ? 1u : what[u] == 2 ? 0x10000u : 0u;
            if (src && kept && j < e.n_keep) src[j] = j;
        }
        const uint32_t before = evict_scan(mine, sums, &total);
        uint32_t f = n_free + (before & 0xffffu), m = n_late + (before >> 16);
        n_free += total & 0xffffu;
        n_late += total >> 16;
        for (int u = 0; u < 4; ++u) {
            const int j = base + 4 * tid + u;
            if (what[u] == 1) e.to[(size_t)rowi * e.move_cap + f++] = j;
            if (what[u] == 2) e.from[(size_t)rowi * e.move_cap + m++] = j;
        }
    }
    if (tid == 0) e.moves[rowi] = (int32_t)n_free;
}

// grid (x, rows): the rows of K and V, positions and weights of the moving slots; then the length
template <typename T>
__global__ __launch_bounds__(256) void paged_evict_move_kernel(PagedCache a, EvictArgs e, T* __restrict__ Kp, T* __restrict__ Vp, int32_t* seq_len,
                                                               int D)
{
    constexpr int VEC = elem<T>::vec;
    const int rowi = blockIdx.y, b = rowi / e.lists, list = rowi % e.lists, row = a.H_kv * D;
    const int n = e.moves[rowi];
    if (n < 0) return;
    if (blockIdx.x == 0 && list == 0 && threadIdx.x == 0) seq_len[b] = e.n_keep;
    const int32_t *from = e.from + (size_t)rowi * e.move_cap, *to = e.to + (size_t)rowi * e.move_cap;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        const size_t r = (size_t)rowi * a.cap;
        e.pos[r + to[i]] = e.pos[r + from[i]];
        e.weights[r + to[i]] = e.weights[r + from[i]];
        if (e.src) e.src[(size_t)rowi * e.n_keep + to[i]] = from[i];
    }
    const int pieces = (e.lists == 1 ? row : D) / VEC, off = e.lists == 1 ? 0 : list * D;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)n * pieces; i += (int64_t)gridDim.x * 256) {
        const int m = (int)(i / pieces), pc = (int)(i - (int64_t)m * pieces);
        const int64_t x = paged_row(a, b, from[m], row), y = paged_row(a, b, to[m], row);
        if (x < 0 || y < 0) continue;
        const int64_t o = off + pc * VEC;
        const u32x4 k = ld16(Kp + x + o), v = ld16(Vp + x + o);
        *reinterpret_cast<u32x4*>(Kp + y + o) = k;
        *reinterpret_cast<u32x4*>(Vp + y + o) = v;
    }
}

__global__ __launch_bounds__(256) void paged_clear_kernel(uint32_t* count, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) count[i] = 0u;
}

}  // namespace sals
