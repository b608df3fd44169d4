// Paged full-rank key-value cache: append of new tokens, attention of one new token per sequence, eviction of tokens by
// accumulated attention weight.
//
// Slot j of sequence b is row j % page_size of page table[b, j / page_size]; a row holds [H_kv, D] elements, K already rotated.
#pragma once
#include "common.hpp"

#include <type_traits>

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

// cos / sin of position * theta^(-2 pair / D): the angle in turns, in fp64, less its whole part (what is left is exact to
// 1e-16 * position turns); cos and sin of its fp32 value, and one step of their series for what that leaves out.
template <int D> __device__ __forceinline__ double rope_frequency(int pair, double log2_theta)   // turns per position
{
    return exp2(-(double)pair * (2.0 / D) * log2_theta) * kInvTwoPi;
}
__device__ __forceinline__ float2 rope_turn(int position, double frequency)
{
    const double t = (double)position * frequency;
    const double part = t - rint(t);
    const float f = (float)part, rest = (float)((part - (double)f) * (1.0 / kInvTwoPi));
    float s, c;
    sincospif(2.f * f, &s, &c);
    return make_float2(fmaf(-rest, s, c), fmaf(rest, c, s));
}

// element offset of slot j's row, or -1 where its page is not there
__device__ __forceinline__ int64_t paged_row(const PagedCache& a, int b, int j, int row)
{
    const uint32_t pg = page_of((uint32_t)j, a.page_mul);
    const int32_t id = a.table[(size_t)b * a.max_pages + pg];
    return (uint32_t)id < (uint32_t)a.n_pages ? (int64_t)id * a.page_stride + (int64_t)(j - (int)pg * a.page_size) * row : -1;
}

// ---- append ---------------------------------------------------------------------------------------------------------------------
// A stream of 4 H_kv D elements a token.  A workgroup takes `tok` consecutive new tokens of a sequence, all heads: cos / sin of its
// tokens once into LDS, then 16-byte pieces, each of K with its partners' piece (which another lane of the wave asks for as well).  The
// last of a sequence's workgroups advances the length: by then all have read it.  It counts behind the pieces: 500 workgroups of 8 tokens
// that counted first queued up at the one address (4001 tokens x 6: 60 us, behind 52, 32 tokens each 41).  The rows are stored
// past the caches, which hold the partners' pieces instead: 41 -> 33 (4.8 TB/s, what a copy reaches).
constexpr int kAppTok = 32;   // tokens of a workgroup at most; fewer as long as there are not three workgroups for each compute unit

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedCache a, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                           const int32_t* __restrict__ q_pos, T* __restrict__ Kp, T* __restrict__ Vp,
                                                           int32_t* seq_len, uint32_t* count, const int32_t* __restrict__ n_new, int n_tok, int tok,
                                                           int32_t* __restrict__ pos, float* __restrict__ weights, int lists, double log2_theta,
                                                           int style)
{
    constexpr int VEC = elem<T>::vec, NP = D / 2, PIECES = D / VEC;
    __shared__ float2 sCS[kAppTok][NP];
    __shared__ int64_t sRow[kAppTok];
    const int b = blockIdx.y, t0 = blockIdx.x * tok, tid = threadIdx.x;
    const int have = min(max(seq_len[b], 0), a.cap);
    const int want = n_new ? min(max(n_new[b], 0), n_tok) : n_tok;
    const int n = min(want, a.cap - have);          // tokens that fit
    const int nt = min(tok, n - t0);
    const int row = a.H_kv * D;
    const uint32_t qp = (uint32_t)q_pos[b];         // (positions past 2^31 wrap)
    for (int i = tid; i < nt * NP; i += 256) sCS[i / NP][i % NP] = rope_turn((int)(qp + t0 + i / NP), rope_frequency<D>(i % NP, log2_theta));
    if (tid < nt) sRow[tid] = paged_row(a, b, have + t0 + tid, row);
    __syncthreads();
    for (int i = tid; i < nt * lists; i += 256) {
        const int list = idiv(i, nt), t = i - list * nt;
        const size_t at = ((size_t)b * lists + list) * a.cap + have + t0 + t;
        pos[at] = (int32_t)(qp + t0 + t);
        weights[at] = 0.f;
    }
    const int pieces = a.H_kv * PIECES;             // of a token
    for (int i = tid; i < nt * pieces; i += 256) {
        const int t = idiv(i, pieces), pc = i - t * pieces;
        const int64_t at = sRow[t];
        if (at < 0) continue;
        const size_t from = ((size_t)b * n_tok + t0 + t) * row + (size_t)pc * VEC;
        // a piece of K, the piece of its partners (itself where neighbours are pairs, half a head away otherwise), a piece of V
        const int ch = pc % PIECES * VEC;
        const bool first = ch < NP;
        const u32x4 kx = ld16(k_new + from), ky = style ? kx : ld16(k_new + (first ? from + NP : from - NP)), v = ld16(v_new + from);
        float x[VEC], y[VEC], r[VEC];
        elem<T>::unpack(kx, x);
        elem<T>::unpack(ky, y);
        if (style) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const float2 cs = sCS[t][(ch + e) / 2];
                r[e] = fmaf(x[e], cs.x, -(x[e + 1] * cs.y));
                r[e + 1] = fmaf(x[e + 1], cs.x, x[e] * cs.y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float2 cs = sCS[t][(ch + e) % NP];
                r[e] = fmaf(x[e], cs.x, first ? -(y[e] * cs.y) : y[e] * cs.y);
            }
        }
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) w[e] = (uint32_t)f32_to_bf16(r[2 * e]) | (uint32_t)f32_to_bf16(r[2 * e + 1]) << 16;
            else w[e] = __float_as_uint(r[e]);
        }
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(Kp + at + (size_t)pc * VEC));
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(Vp + at + (size_t)pc * VEC));
    }
    if (tid == 0 && (gridDim.x == 1 || arrive(count + b, gridDim.x) == gridDim.x - 1) && n > 0) seq_len[b] = have + n;
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
// softmax over a sequence's slots in one pass over K and V, the work split over the slots of the whole batch.
//
// Work.  A sequence of S slots is ceil(S / TB) blocks of TB slots (at least one, so that somebody writes its output); the blocks of
// all sequences, one behind the other, are dealt in equal consecutive shares to the workgroups of a KV head.  A share may begin and
// end inside a sequence and hold whole ones, so a ragged batch loads the chip as evenly as an even one.  What a workgroup finds of a
// sequence that others share goes to the workspace, and the last of them to arrive joins the pieces in the order of the shares.
//
// Matrix cores.  A wave takes a block at a time, for up to 16 query heads of a KV head (the columns):
//   S^T = K q^T      rows = slots, contraction over channels: a lane's 16 bytes of a K row are an operand as they lie in memory
//   O^T += V^T p^T   rows = channels, contraction over slots: the lane that holds the weights of slots c CH .. c CH + CH - 1 of head n
//                    (the layout that S^T leaves, with the slots of K's rows dealt accordingly) needs the same slots of channel n of V;
//                    it loads 16 (8) bytes of each of their rows and byte permutes turn them, so nothing passes through LDS.
// bf16: the rotated query is three bf16 pieces (exact to fp32's own rounding), and so is a weight (split3); products and sums fp32.
// No piece is zero unless the number is, and all have its sign: infinite keys and values stay what they are.  (With two pieces, 16 bits of a weight, outputs were off
// by 3e-6 before their rounding, ten times what the sums take.)
// A maximum is followed only when a logit exceeds it by more than 8 (in units of ln 2; weights then stay below 2^8), which few blocks need.
constexpr int kPgHeads = 16;           // query heads of a workgroup
constexpr int kPgWaves = 8;
constexpr int kPgGroups = 256;         // workgroups: one per compute unit
constexpr int kPgKept = 2048;          // floats of logits that a wave keeps
constexpr int kPgAhead = 8;            // pieces of a shared sequence that a thread requests together

template <typename T> struct PgBlock;
template <> struct PgBlock<bf16_t> { static constexpr int TB = 32; };
template <> struct PgBlock<float> { static constexpr int TB = 16; };

struct PagedWork {
    int blocks, shares, q, r;     // of all sequences; workgroups of a head; the first r shares have q + 1 blocks, the others q
    __device__ __forceinline__ int begin(int w) const { return w * q + min(w, r); }
    __device__ __forceinline__ int share(int x) const   // the one that block x belongs to
    {
        const int split = r * (q + 1);
        return x < split ? per_share(x, q + 1) : r + per_share(x - split, q);
    }
    // x / d; 24 bits divide in half the instructions
    __device__ __forceinline__ int per_share(int x, int d) const { return blocks < 1 << 24 ? idiv(x, d) : (int)((uint32_t)x / (uint32_t)d); }
};

// Pieces of shared sequences: 2 w of share w for one that began before it, 2 w + 1 for one that begins in it.
struct PagedParts {
    float* sum;                   // [2 shares][workgroups side by side][KV heads of one][rows][D]
    float2* stat;                 // [2 shares][workgroups side by side][KV heads of one][rows]: maximum, sum
    uint32_t* count;              // [B][workgroups side by side], zero between launches
    float2* final_stat;           // [B * H]: maximum, 1 / sum
    int rows;                     // query heads of a KV head in a workgroup, at most
};

// Stores and loads that pass the caches of the compute unit and of its die, for what one workgroup leaves to another of the same
// launch: ordinary ones would need a write-back and an invalidation of a whole L2 around them.  A workgroup's stores
// are done, for every workgroup of the device, behind device_stores_done() in every thread and a barrier.
__device__ __forceinline__ f32x4 ld4_device(const float* p)
{
    const uint64_t* u = reinterpret_cast<const uint64_t*>(p);
    const uint64_t a = __hip_atomic_load(u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), b = __hip_atomic_load(u + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return f32x4{__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32)), __uint_as_float((uint32_t)b), __uint_as_float((uint32_t)(b >> 32))};
}
__device__ __forceinline__ void st4_device(float* p, const f32x4& v)
{
    uint64_t* u = reinterpret_cast<uint64_t*>(p);
    __hip_atomic_store(u, (uint64_t)__float_as_uint(v.y) << 32 | __float_as_uint(v.x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(u + 1, (uint64_t)__float_as_uint(v.w) << 32 | __float_as_uint(v.z), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 ld2_device(const float2* p)
{
    const uint64_t a = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32)));
}
__device__ __forceinline__ void st2_device(float2* p, float2 v)
{
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)__float_as_uint(v.y) << 32 | __float_as_uint(v.x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// x >= 0 as three floats of 8 significant bits: its sum exactly, every piece above zero where x is (from 2^-95 on).  Pieces are cut off from
// what is one step below, so that something is left of a power of two, or of any number that has the piece's bits alone.  The upper
// halves are the pieces in bf16 (the lower halves of the first two are to be dropped).
struct Split3 { uint32_t x0, x1, x2; };
__device__ __forceinline__ Split3 split3(float x)
{
    Split3 s;
    s.x0 = __builtin_elementwise_sub_sat(__float_as_uint(x), 1u);
    const float r = x - __uint_as_float(s.x0 & 0xffff0000u);
    s.x1 = __builtin_elementwise_sub_sat(__float_as_uint(r), 1u);
    s.x2 = __float_as_uint(r - __uint_as_float(s.x1 & 0xffff0000u));
    return s;
}
__device__ __forceinline__ uint32_t upper_halves(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302); }

__device__ __forceinline__ void device_stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// a barrier for what was written to LDS; loads on their way stay there
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ float max_xor_rows(float v)   // over the four lanes that hold a head
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_xor_rows(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// grid: a workgroup for each compute unit (see `lg` for which work it gets); logits: null, or [B * H][logit_stride] to be left,
// keep: the LDS for runs of them is there
template <typename T, int D, bool WHOLE>   // WHOLE: the CH slots of a lane lie in one page
__global__ __launch_bounds__(kPgWaves * 64, 2) void paged_attend_kernel(const int32_t* __restrict__ seq_len, int B, int cap, int kv_heads, int tiles,
                                                                       PagedCache a, const T* __restrict__ q, const int32_t* __restrict__ q_pos,
                                                                       const T* __restrict__ Kp, const T* __restrict__ Vp, T* __restrict__ out,
                                                                       PagedParts parts, float* __restrict__ logits, int logit_stride, int keep,
                                                                       float scale, double log2_theta, int style)
{
    constexpr bool BF = sizeof(T) == 2;
    constexpr int TB = PgBlock<T>::TB, CH = TB / 4, VEC = elem<T>::vec;
    constexpr int NKT = TB / 16;               // row tiles of S^T
    constexpr int NS = D / (4 * VEC);          // 16-byte pieces of a K row per lane
    constexpr int NJ = D / 16;                 // row tiles of O^T
    constexpr int VW = NJ * sizeof(T) / 4;     // 32-bit words of a V row per lane
    constexpr int NID = WHOLE ? 1 : CH, NIK = WHOLE ? 1 : NKT;
    constexpr int LROW = D + 4;
    constexpr int THREADS = kPgWaves * 64;
    extern __shared__ __attribute__((aligned(16))) float sO[];   // [kPgWaves][parts.rows][LROW], then the factors of pieces
    __shared__ u32x4 sQ[2][BF ? 3 : 1][NS][64];   // the query as the matrix instructions take it
    __shared__ float sM[kPgWaves][kPgHeads], sL[kPgWaves][kPgHeads];
    __shared__ __attribute__((aligned(16))) f32x4 sX[THREADS];
    __shared__ uint32_t sLast;

    const int tid0 = threadIdx.x, wave = wave_uniform(tid0 >> 6);
    // ---- this workgroup's share ----
    const int per = (B + 63) >> 6;           // sequences of a lane; with one, their lengths stay in the lanes
    auto clamped = [&](int n) { return min(max(n, 0), cap); };
    auto blocks_in = [&](int n) { return max(1, (n + TB - 1) / TB); };
    uint32_t mine = 0;
    int lane_len = 0;
    const int lane0 = tid0 & 63;
    for (int i = 0; i < per; ++i)
        if (lane0 * per + i < B) {
            lane_len = clamped(seq_len[lane0 * per + i]);
            mine += (uint32_t)blocks_in(lane_len);
        }
    // (while the lengths are on their way)
    const double frequency = rope_frequency<D>(tid0 & (D / 2 - 1), log2_theta);
    const int row = a.H_kv * D;
    const uint32_t upto = wave_incl_scan(mine);
    PagedWork W;
    W.blocks = __builtin_amdgcn_readlane((int)upto, 63);
    // Two neighbouring KV heads of a workgroup, four waves for each, read longer pieces of memory, and the channels that are slow for every
    // fourth 256 bytes are shared out; a sequence then has twice as many pieces to join.  Worth it from 16 blocks for each workgroup on,
    // where a sequence has no more than about 16 pieces or is long (32 heads, 16 x 4096 slots: 177 -> 165 us; 8 heads, 8 x 8191: 51.7 ->
    // 50.0; 32 of 188 to 6002: 76.7 -> 71.8; 1 x 4100: 12.8, with two 18.0; 1 x 32768: 28.2, with two 32.2).  Four with two waves each: 172,
    // and no faster for heads of 64 channels.
    const int single = kv_heads * tiles, per_group = idiv(kPgGroups, single);
    const int lg = tiles == 1 && !(kv_heads & 1) && W.blocks >= 16 * per_group && (2 * per_group <= 16 * B || W.blocks >= 128 * per_group) ? 1 : 0;
    const int HPW = 1 << lg, WPH = kPgWaves >> lg, heads = single >> lg;
    W.shares = min(max(1, idiv(kPgGroups, heads)), W.blocks);
    // Workgroup -> share and KV heads.  Tiles of 16 query heads that read the same rows lie 8 apart, on one die and its L2.
    int w, hg;
    if (tiles == 1) {
        w = idiv(blockIdx.x, heads);
        hg = blockIdx.x - w * heads;
    } else {
        const int eight = idiv(blockIdx.x >> 3, tiles), c = eight * 8 + (blockIdx.x & 7);
        w = idiv(c, kv_heads);
        hg = (c - w * kv_heads) * tiles + (blockIdx.x >> 3) - eight * tiles;
    }
    if (w >= W.shares) return;
    // A sequence that begins in a share costs it the end of one stream and the start of another, as much as some blocks, which are dealt
    // with the real ones: up to 4 (up to 1, 2, 4, 8 and 16 of them: 32 sequences of 188 to 6002 slots 74.6, 73.2, 72.4, 75.6 and 77.7 us, 256
    // of up to 800 slots 87.6, 86.4, 86.6, 88.6 and 92.7); not where all are equally long and whole numbers of shares (8 x 8191 slots:
    // 50.0, with them 51.2).
    int pad = 0;
    W.q = W.per_share(W.blocks, W.shares);
    if (W.q >= 8) {
        const bool even = per == 1 && wave_min_u32(lane0 < B ? mine : 0xffffffffu) == wave_max_u32(mine) && W.shares - idiv(W.shares, B) * B == 0;
        if (!even) {
            pad = min(4, W.q / 8);
            W.blocks += pad * B;
            W.q = W.per_share(W.blocks, W.shares);
        }
    }
    W.r = W.blocks - W.q * W.shares;
    // a workgroup's query heads are consecutive, nh for each of its KV heads
    const int sub = wave >> (3 - lg), H = a.H_kv * a.group;
    const int g = tiles == 1 ? hg * HPW + sub : idiv(hg, tiles);
    const int first_head = tiles == 1 ? hg * HPW * a.group : g * a.group + (hg - g * tiles) * kPgHeads;
    const int nh = min(kPgHeads, (g + 1) * a.group - first_head - sub * a.group), h0 = first_head + sub * a.group;
    const int wave_of = wave & (WPH - 1);   // of the KV head
    int at = W.begin(w);
    const int end = W.begin(w + 1);
    const int first_lane = __popcll(__ballot(upto + (uint32_t)(pad * min(B, (lane0 + 1) * per)) <= (uint32_t)at));
    int b = first_lane * per, base = __builtin_amdgcn_readlane((int)(upto - mine), first_lane) + pad * b;
    auto length_of = [&](int s) { return per == 1 ? __builtin_amdgcn_readlane(lane_len, s) : wave_uniform(clamped(seq_len[s])); };
    for (int n; base + (n = pad + blocks_in(length_of(b))) <= at; ++b) base += n;

    for (bool again = false; at < end; again = true) {
        if (again) __syncthreads();   // (LDS is taken anew)
        // (new values for the compiler: what follows from them is computed where it is wanted, not kept through the stream)
        int tid = tid0;
        asm volatile("" : "+v"(tid));
        int lane = tid & 63, n16 = lane & 15, c4 = lane >> 4;
        const int S = length_of(b), n_blocks = pad + blocks_in(S);
        const bool begins = at == base;
        const int blk0 = max(0, at - base - pad), blk1 = min(end - base, n_blocks) - pad, live1 = min(blk1, (S + TB - 1) / TB);
        const int32_t* tb = a.table + (size_t)b * a.max_pages;

        // ---- pages and rows of a block ----
        struct Ids { int32_t k[NIK], v[NID]; };
        auto k_slot = [&](int t0, int t) { return WHOLE ? t0 + (n16 >> 2) * CH : min(t0 + (n16 >> 2) * CH + t * 4 + (n16 & 3), S - 1); };
        auto v_slot = [&](int t0, int e) { return WHOLE ? t0 + c4 * CH : min(t0 + c4 * CH + e, S - 1); };
        // a run of CH slots that begins past the end re-reads the last one that does not
        auto held = [&](int j) { return WHOLE ? min(j, (S - 1) & ~(CH - 1)) : j; };
        auto load_ids = [&](Ids& I, int blk) {
            const int t0 = min(blk, live1 - 1) * TB;
#pragma unroll
            for (int t = 0; t < NIK; ++t) I.k[t] = tb[page_of((uint32_t)held(k_slot(t0, t)), a.page_mul)];
#pragma unroll
            for (int e = 0; e < NID; ++e) I.v[e] = tb[page_of((uint32_t)held(v_slot(t0, e)), a.page_mul)];
        };
        // element offset of slot j's row; a page that is not there is read as page 0, and masked
        auto row_at = [&](int32_t id, int j) {
            const uint32_t pg = page_of((uint32_t)j, a.page_mul);
            const uint32_t page = (uint32_t)id < (uint32_t)a.n_pages ? (uint32_t)id : 0u;
            return (int64_t)page * a.page_stride + (int64_t)(uint32_t)((j - (int)pg * a.page_size) * row);
        };
        u32x4 K[NKT][NS];
        uint32_t V[CH][VW];
        auto load_k = [&](const Ids& I, int blk) {
            const int t0 = blk * TB;
#pragma unroll
            for (int t = 0; t < NKT; ++t) {
                const int j = held(k_slot(t0, t));
                const T* p = Kp + row_at(I.k[WHOLE ? 0 : t], j) + (WHOLE ? (t * 4 + (n16 & 3)) * row : 0) + g * D + c4 * VEC;
#pragma unroll
                for (int s = 0; s < NS; ++s) K[t][s] = ld16(p + s * 4 * VEC);
            }
        };
        auto load_v = [&](const Ids& I, int blk) {
            const int t0 = blk * TB;
            const T* p0 = nullptr;
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                if (!WHOLE || e == 0) p0 = Vp + row_at(I.v[WHOLE ? 0 : e], held(v_slot(t0, e))) + g * D;
                const T* p = WHOLE ? p0 + e * row : p0;
                if constexpr (BF && VW == 2) {
                    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p + n16 * NJ));
                    V[e][0] = x.x; V[e][1] = x.y;
                } else {
#pragma unroll
                    for (int h = 0; h < VW / 4; ++h) {   // fp32: pieces of 4 channels, 64 channels apart
                        const u32x4 x = ld16_stream(p + h * 64 + n16 * VEC);
                        V[e][4 * h] = x.x; V[e][4 * h + 1] = x.y; V[e][4 * h + 2] = x.z; V[e][4 * h + 3] = x.w;
                    }
                }
            }
        };

        // the query and its position come with the table's entries, which the first rows wait for: it is rotated while those are on their way
        int blk = blk0 + wave_of;
        // a thread's pair of channels in some of the 16 columns of every KV head (columns without a query head are zero)
        constexpr int COLS = THREADS / (D / 2), NQ = 2 * kPgHeads / COLS;
        const int pair = tid % (D / 2), ch1 = style ? 2 * pair : pair, ch2 = style ? 2 * pair + 1 : pair + D / 2;
        const int position_v = ld_uniform_i32(q_pos + b);
        typedef typename std::conditional<BF, uint16_t, uint32_t>::type Raw;
        uint32_t q1[NQ], q2[NQ];   // bits; not set to anything first: behind a branch a value that is one of two would be waited for there
#pragma unroll
        for (int k = 0; k < NQ; ++k) {
            asm volatile("" : "=v"(q1[k]), "=v"(q2[k]));
            const int col = tid / (D / 2) + k * COLS, h = col % kPgHeads;
            if (h < nh && col < HPW * kPgHeads) {
                const Raw* p = reinterpret_cast<const Raw*>(q) + ((size_t)b * H + first_head + col / kPgHeads * nh + h) * D;
                q1[k] = p[ch1];
                q2[k] = p[ch2];
            }
        }
        Ids I0, I1;
        if (blk < live1) {
            load_ids(I0, blk);
            load_ids(I1, blk + WPH);
        }
        // (vmcnt(0), the other counters left alone: all of these are one trip to memory, and behind it the compiler knows that the query is
        // there; it would wait for the rows with it otherwise)
        __builtin_amdgcn_s_waitcnt(0x0f70);
        if (blk < live1) {
            load_k(I0, blk);
            load_v(I0, blk);
        }

        // the shares that this sequence is spread over
        const bool ends = blk1 == n_blocks - pad, alone = begins && ends;
        const int w0 = begins ? w : W.share(base), w1 = ends ? w : W.share(base + n_blocks - 1);

        // ---- the rotated query of these heads, scaled ----
        {
            const float2 cs = rope_turn(position_v, frequency);
#pragma unroll
            for (int k = 0; k < NQ; ++k) {
                const int col = tid / (D / 2) + k * COLS;
                if (col >= HPW * kPgHeads) break;
                const bool live = col % kPgHeads < nh;
                const float x = live ? __uint_as_float(q1[k] << (BF ? 16 : 0)) : 0.f, y = live ? __uint_as_float(q2[k] << (BF ? 16 : 0)) : 0.f;
                const float r[2] = {fmaf(x, cs.x, -(y * cs.y)) * scale, fmaf(y, cs.x, x * cs.y) * scale};
                const int ch[2] = {ch1, ch2};
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t piece[3] = {__float_as_uint(r[u]), 0u, 0u};
                    if constexpr (BF) {   // (pieces of the element's sign, none of them zero: an infinite key stays one)
                        const Split3 s = split3(fabsf(r[u]));
                        const uint32_t sign = __float_as_uint(r[u]) & 0x80000000u;
                        piece[0] = (s.x0 | sign) >> 16; piece[1] = (s.x1 | sign) >> 16; piece[2] = (s.x2 | sign) >> 16;
                    }
#pragma unroll
                    for (int k3 = 0; k3 < (BF ? 3 : 1); ++k3)
                        reinterpret_cast<Raw*>(&sQ[col / kPgHeads][k3][ch[u] / (4 * VEC)][ch[u] / VEC % 4 * 16 + col % kPgHeads])[ch[u] % VEC] = (Raw)piece[k3];
                }
            }
        }
        lds_barrier();

        // ---- the stream ----
        float m = -INFINITY, l = 0.f;
        f32x4 O[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) O[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // Logits that are wanted are kept in LDS and leave in runs, where a wave has more than two blocks: a few bytes stored beside every
        // block slow the stream down (with the weights' launch, 16 x 4096 slots of 32 heads 201 -> 189 us, 8 x 8191 of 8 64 -> 61).
        float* const kept = sO + wave * kPgKept;
        const int keep_most = keep && live1 - blk0 > 2 * WPH ? idiv(kPgKept / TB, nh) : 0;
        int n_kept = 0;   // blocks, `blk` the last one
        auto leave = [&]() {
            constexpr int PL = TB / 4;
            const int first = blk - (n_kept - 1) * WPH;
            for (int i = lane; i < n_kept * nh * PL; i += kWave) {
                const int line = i / PL, k = idiv(line, nh), h = line - k * nh;
                const f32x4 v = *reinterpret_cast<const f32x4*>(kept + i * 4);
                *reinterpret_cast<f32x4*>(logits + ((size_t)b * H + h0 + h) * logit_stride + (size_t)(first + k * WPH) * TB + i % PL * 4) = v;
            }
            n_kept = 0;
        };
        // MORE: the block behind is requested.  (No branch around its loads: the compiler would wait for all that are under way, not
        // knowing which ones are.)
        auto block = [&](auto MORE) {
            const int t0 = blk * TB;
            constexpr int CHAINS = BF ? 1 : 4;   // fp32: sums of a quarter of the channels each, whose roundings add up less
            f32x4 x[NKT > CHAINS ? NKT : CHAINS];
#pragma unroll
            for (int t = 0; t < (BF ? NKT : CHAINS); ++t) x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            int at_lane = lane;
            asm volatile("" : "+v"(at_lane));   // (read from LDS for every block: the registers are wanted for rows)
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int k = (BF ? 2 : 0); k >= 0; --k) {
                    const u32x4 qv = sQ[sub][k][s][at_lane];
#pragma unroll
                    for (int t = 0; t < NKT; ++t) {
                        if constexpr (BF) {
                            x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, K[t][s]), __builtin_bit_cast(bf16x8, qv), x[t], 0, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                x[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(K[t][s][e]), __uint_as_float(qv[e]), x[e], 0, 0, 0);
                        }
                    }
                }
            if constexpr (!BF) x[0] = (x[0] + x[1]) + (x[2] + x[3]);
            // which of this lane's slots count (slot t0 + CH c4 + e is x[e / 4][e % 4])
            bool whole = t0 + TB <= S;
#pragma unroll
            for (int e = 0; e < NID; ++e) whole = whole && (uint32_t)I0.v[e] < (uint32_t)a.n_pages;
            if (__ballot(!whole)) {
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    const bool ok = t0 + c4 * CH + e < S && (uint32_t)I0.v[WHOLE ? 0 : e] < (uint32_t)a.n_pages;
                    if (!ok) x[e >> 2][e & 3] = -INFINITY;
                }
            }
            const uint64_t part_of = __ballot(!whole);
            Ids I2;
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (MORE()) {
                load_ids(I2, blk + 2 * WPH);
                load_k(I1, blk + WPH);
            }
            float top = x[0][0];
#pragma unroll
            for (int e = 1; e < CH; ++e) top = fmaxf(top, x[e >> 2][e & 3]);
            if (__ballot(top > m + 8.f)) {   // (also the first time: m is -infinity)
                const float mn = fmaxf(m, max_xor_rows(top));
                const float f = mn > -INFINITY ? __builtin_amdgcn_exp2f(m - mn) : 1.f;
                m = mn;
                l *= f;
#pragma unroll
                for (int j = 0; j < NJ; ++j) O[j] *= f;
            }
            const float ref = m > -INFINITY ? m : 0.f;   // (nothing yet: all are -infinity)
            float p[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                p[e] = __builtin_amdgcn_exp2f(x[e >> 2][e & 3] - ref);
                l += p[e];
            }
            if (part_of) {   // what lies in slots that do not count may be anything
#pragma unroll
                for (int e = 0; e < CH; ++e) {
                    const bool ok = t0 + c4 * CH + e < S && (uint32_t)I0.v[WHOLE ? 0 : e] < (uint32_t)a.n_pages;
#pragma unroll
                    for (int k = 0; k < VW; ++k) V[e][k] = ok ? V[e][k] : 0u;
                }
            }
            if constexpr (BF) {
                u32x4 pw[3];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const Split3 a0 = split3(p[2 * k]), a1 = split3(p[2 * k + 1]);
                    pw[0][k] = upper_halves(a0.x0, a1.x0);
                    pw[1][k] = upper_halves(a0.x1, a1.x1);
                    pw[2][k] = upper_halves(a0.x2, a1.x2);
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    u32x4 v;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = __builtin_amdgcn_perm(V[2 * k + 1][j >> 1], V[2 * k][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
                    for (int k = 2; k >= 0; --k)
                        O[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pw[k]), O[j], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int e = 0; e < CH; ++e)
#pragma unroll
                    for (int j = 0; j < NJ; ++j) O[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(V[e][j]), p[e], O[j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);   // (the rows behind take these registers, not others)
            if constexpr (MORE()) {
                load_v(I1, blk + WPH);
                I0 = I1;
                I1 = I2;
            }
            if (keep_most > 0) {
                if (n16 < nh)
#pragma unroll
                    for (int t = 0; t < NKT; ++t) *reinterpret_cast<f32x4*>(kept + (n_kept * nh + n16) * TB + c4 * CH + 4 * t) = x[t];
                if (++n_kept == keep_most) leave();
            } else if (logits && n16 < nh) {
                float* to = logits + ((size_t)b * H + h0 + n16) * logit_stride + t0 + c4 * CH;
#pragma unroll
                for (int t = 0; t < NKT; ++t) *reinterpret_cast<f32x4*>(to + 4 * t) = x[t];
            }
        };
        for (; blk + WPH < live1; blk += WPH) block(std::true_type{});
        if (blk < live1) block(std::false_type{});
        if (keep_most > 0) {   // (what is kept lies where the waves' sums come next)
            leave();
            lds_barrier();
        }

        // ---- the waves joined ----
        asm volatile("" : "+v"(tid));
        lane = tid & 63; n16 = lane & 15; c4 = lane >> 4;
        const int n_live = min(WPH, live1 - blk0);        // waves of a KV head that had a block
        if (wave_of < n_live) {
            l = sum_xor_rows(l);
            if (lane < kPgHeads) { sM[wave][lane] = m; sL[wave][lane] = l; }
            // channel of O[j][i] of this lane
            auto channel = [&](int j, int i) { return BF ? (c4 * 4 + i) * NJ + j : (j >> 2) * 64 + (c4 * 4 + i) * 4 + (j & 3); };
            if (n16 < nh)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < NJ; j += 4)
                        *reinterpret_cast<f32x4*>(sO + (wave * parts.rows + n16) * LROW + channel(j, i)) =
                            f32x4{O[j][i], O[j + 1][i], O[j + 2][i], O[j + 3][i]};
        }
        __syncthreads();
        // four channels of a head at a time: quad -> (KV head, query head, channels)
        const int quads = HPW * nh * (D / 4);
        auto finish = [&](int quad, f32x4 A, float Mh, float L) {
            const size_t h = (size_t)b * H + first_head + quad / (D / 4);
            const float inv = L != 0.f ? 1.f / L : 0.f;   // (nothing attended: zero)
            const f32x4 y = A * inv;
            T* to = out + h * D + quad % (D / 4) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) elem<T>::store(to + e, y[e]);
            if (quad % (D / 4) == 0) parts.final_stat[h] = make_float2(L != 0.f ? Mh : 0.f, inv);
        };
        const size_t piece = ((size_t)(2 * w + begins) * heads + hg) * (HPW * parts.rows);
        for (int quad = tid; quad < quads; quad += THREADS) {
            const int hh = quad / (D / 4), s = hh >= nh ? 1 : 0, h = hh - s * nh;
            float mv[kPgWaves], lv[kPgWaves];
            f32x4 ov[kPgWaves];
#pragma unroll
            for (int v = 0; v < kPgWaves; ++v) {
                const int wv = min(s * WPH + v, kPgWaves - 1);
                mv[v] = v < n_live ? sM[wv][h] : -INFINITY;   // (the others left nothing)
                lv[v] = sL[wv][h];
                ov[v] = *reinterpret_cast<const f32x4*>(sO + (wv * parts.rows + h) * LROW + quad % (D / 4) * 4);
            }
            float Mh = mv[0], L = 0.f;
            f32x4 A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 1; v < kPgWaves; ++v) Mh = fmaxf(Mh, mv[v]);
#pragma unroll
            for (int v = 0; v < kPgWaves; ++v)
                if (v < n_live) {   // (a sum of weight zero counts too: what is not finite in it is to stay)
                    const float f = lv[v] != 0.f ? __builtin_amdgcn_exp2f(mv[v] - Mh) : 0.f;
                    L = fmaf(lv[v], f, L);
                    A += ov[v] * f;
                }
            if (alone) {
                finish(quad, A, Mh, L);
            } else {
                st4_device(parts.sum + (piece + hh) * D + quad % (D / 4) * 4, A);
                if (quad % (D / 4) == 0) st2_device(parts.stat + piece + hh, make_float2(Mh, L));
            }
        }
        if (!alone) {
            // the pieces are where the whole device sees them before this workgroup counts as arrived
            device_stores_done();
            __syncthreads();
            if (tid == 0) sLast = arrive(parts.count + (size_t)b * heads + hg, (uint32_t)(w1 - w0 + 1)) == (uint32_t)(w1 - w0);
            __syncthreads();
            if (sLast) {
                asm volatile("" : "+v"(tid));
                lane = tid & 63;
                // (share, kind) of the pieces: the first share's goes on behind it, the others' began before
                auto piece_of = [&](int v) { return ((size_t)(2 * v + (v == w0)) * heads + hg) * (HPW * parts.rows); };
                const int n = w1 - w0 + 1;
                // the statistics of a head are a wave's: the first of them, then this thread's first sums, then what follows from the former
                auto stat_of = [&](int hh, int v) { return v < n ? ld2_device(parts.stat + piece_of(w0 + v) + hh) : make_float2(-INFINITY, 0.f); };
                float2 st = make_float2(-INFINITY, 0.f);
                if (wave < HPW * nh) st = stat_of(wave, lane);
                // with fewer quads than threads several threads share a quad's pieces
                const int sharers = quads < THREADS ? idiv(THREADS, quads) : 1, mine_of = sharers > 1 ? idiv(tid, quads) : 0;
                f32x4 x[kPgAhead];
                auto request = [&](int quad, int v) {
#pragma unroll
                    for (int u = 0; u < kPgAhead; ++u) {
                        x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                        if (v + u * sharers < n) x[u] = ld4_device(parts.sum + piece_of(w0 + v + u * sharers) * D + quad * 4);
                    }
                };
                int quad = sharers > 1 ? tid - mine_of * quads : tid;
                const bool works = mine_of < sharers && quad < quads;
                if (works) request(quad, mine_of);
                for (int hh = wave; hh < HPW * nh; hh += kPgWaves) {
                    if (hh != wave) st = stat_of(hh, lane);
                    float Mx = wave_max(st.x);
                    for (int v = kWave; v < n; v += kWave) Mx = fmaxf(Mx, wave_max(stat_of(hh, v + lane).x));
                    float L = 0.f;
                    for (int v = 0; v < n; v += kWave) {
                        if (v > 0) st = stat_of(hh, v + lane);
                        const float f = st.y != 0.f ? __builtin_amdgcn_exp2f(st.x - Mx) : 0.f;   // (NaN stays NaN)
                        L = fmaf(st.y, f, L);
                        if (v + lane < n) sO[hh * n + v + lane] = f;
                    }
                    L = wave_sum(L);
                    if (lane == 0) { sM[hh / kPgHeads][hh % kPgHeads] = Mx; sL[hh / kPgHeads][hh % kPgHeads] = L; }
                }
                __syncthreads();
                for (int q0 = 0; q0 < quads; q0 += THREADS, quad += THREADS) {
                    f32x4 A = {0.f, 0.f, 0.f, 0.f};
                    const int hh = quad / (D / 4);
                    if (works && quad < quads) {
                        for (int v = mine_of; v < n; v += kPgAhead * sharers) {
                            if (q0 > 0 || v > mine_of) request(quad, v);
                            float f[kPgAhead];
#pragma unroll
                            for (int u = 0; u < kPgAhead; ++u) f[u] = sO[hh * n + min(v + u * sharers, n - 1)];
#pragma unroll
                            for (int u = 0; u < kPgAhead; ++u)
#pragma unroll
                                for (int e = 0; e < 4; ++e) A[e] = fmaf(x[u][e], f[u], A[e]);   // (x is zero behind the last piece)
                        }
                        if (sharers == 1) finish(quad, A, sM[hh / kPgHeads][hh % kPgHeads], sL[hh / kPgHeads][hh % kPgHeads]);
                    }
                    if (sharers > 1) {
                        sX[tid] = A;
                        __syncthreads();
                        if (tid < quads) {
                            for (int k = 1; k < sharers; ++k) A += sX[tid + k * quads];
                            finish(tid, A, sM[hh / kPgHeads][hh % kPgHeads], sL[hh / kPgHeads][hh % kPgHeads]);
                        }
                    }
                }
            }
        }
        base += n_blocks;
        at = base;
        ++b;
    }
}

// weights[b, list, j] += sum over the list's heads, in their order, of the softmax weight.  grid (x, lists, B); a thread takes four slots
// at a time; its first logits are requested before the length and the statistics are there (the call's second launch: 8 x 8191 slots,
// 32 heads: 5 us).
__global__ __launch_bounds__(256) void paged_weights_kernel(PagedCache a, const float* __restrict__ logits, const float2* __restrict__ stat,
                                                            int logit_stride, float* __restrict__ weights)
{
    constexpr int AHEAD = 4;
    __shared__ float2 sStat[1024];
    const int lists = gridDim.y, b = blockIdx.z, H = a.H_kv * a.group, nh = idiv(H, lists), tid = threadIdx.x;
    const size_t h0 = (size_t)b * H + blockIdx.y * nh;
    const float* const x0 = logits + h0 * logit_stride;
    float* const w = weights + ((size_t)b * lists + blockIdx.y) * a.cap;
    int j = (blockIdx.x * 256 + tid) * 4;
    f32x4 x[AHEAD];
    auto request = [&](int h) {   // (rows of logits go on to a multiple of 32 slots)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) x[u] = *reinterpret_cast<const f32x4*>(x0 + (size_t)min(h + u, nh - 1) * logit_stride + j);
    };
    if (j < a.cap) request(0);
    const int S = min(max(a.seq_len[b], 0), a.cap);
    for (int h = tid; h < nh; h += 256) sStat[h] = stat[h0 + h];
    __syncthreads();
    for (bool first = true; j < S; j += gridDim.x * 1024, first = false) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int h = 0; h < nh; h += AHEAD) {
            if (!first || h > 0) request(h);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (h + u < nh) {
                    const float2 st = sStat[h + u];
#pragma unroll
                    for (int e = 0; e < 4; ++e)   // (slots without a page get nothing, be the others' weights NaN)
                        sum[e] = x[u][e] != -INFINITY ? fmaf(__builtin_amdgcn_exp2f(x[u][e] - st.x), st.y, sum[e]) : sum[e];
                }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < S) w[j + e] += sum[e];
    }
}

// ---- eviction -------------------------------------------------------------------------------------------------------------------
// A list's n_keep slots of the largest keys, and the moves that bring them below slot n_keep.  One workgroup per list; a wave holds
// consecutive slots, 256 at a step (four for each lane), in registers up to 8 steps (tables of 32768 slots; longer ones, and those of more than
// 16384 with few lists, further below).
//
// Threshold: the key and the slot of the last one that stays.  Where up to kEvFew leave they are found one by one (the lowest first).
// Otherwise a histogram over the keys' leading 12 bits (keys are the floats' bits in order, so eight bins for a factor of two) names the
// bin, as a rule of a few dozen, whose members are ranked against each other in LDS; larger ones are split by the next 12 and 8 bits,
// and of one key's slots the first ones stay.  Then the slots in order: which become free below n_keep, which move; the places in
// the lists of moves by one prefix sum.
constexpr int kEvThreads = 1024;
constexpr int kEvWaves = kEvThreads / kWave;
constexpr int kEvBins = 4096;
constexpr int kEvStep = 256;          // slots of a wave at a time
constexpr int kEvChunk = kEvStep * kEvWaves;
constexpr int kEvMembers = 256;
constexpr int kEvFew = 8;
constexpr int kEvFused = 64;          // moves of a list that its workgroup makes itself

struct EvictArgs {
    const int32_t* q_pos;
    int32_t* pos;
    float* weights;
    int32_t *src, *moves, *from, *to;   // moves [rows]: rows to move, -1 for none and no change of the length; from, to [rows, move_cap]
    uint32_t* count;                    // [B], zero between launches
    int lists, n_keep, n_sink, n_recent, move_cap, D;
    int fused;                          // no list has more than kEvFused moves: no second launch
};

// what a slot is ranked by: NaN below all weights, protected ones above all
constexpr uint32_t kEvNan = 0u, kEvProtected = 0xffffffffu;
__device__ __forceinline__ uint32_t evict_key(float w, int32_t p, int32_t n_sink, int64_t recent_from)
{
    return p < n_sink || (int64_t)p > recent_from ? kEvProtected : w != w ? kEvNan : score_key(w);
}

// One wave makes `n` <= 64 moves of a list: rows of K and V (the list's part of them; stored past the caches: an eviction that
// moves 4 x 3700 rows of 2 KB 49 -> 45 us), positions and weights.
template <typename T>
__device__ __forceinline__ void evict_move(const PagedCache& a, const EvictArgs& e, T* Kp, T* Vp, int rowi, const int32_t* from, const int32_t* to, int n)
{
    constexpr int VEC = elem<T>::vec;
    const int lane = lane_id(), b = idiv(rowi, e.lists), list = rowi - b * e.lists, row = a.H_kv * e.D;
    int64_t x = -1, y = -1;   // lane k: move k
    if (lane < n) {
        const int f = from[lane], t = to[lane];
        x = paged_row(a, b, f, row);
        y = paged_row(a, b, t, row);
        const size_t r = (size_t)rowi * a.cap;
        const int32_t p = e.pos[r + f];
        const float w = e.weights[r + f];
        e.pos[r + t] = p;
        e.weights[r + t] = w;
        if (e.src) e.src[(size_t)rowi * e.n_keep + t] = f;
        if (x < 0 || y < 0) x = y = -1;   // a page that is not there
        else if (e.lists > 1) { x += list * e.D; y += list * e.D; }
    }
    const int pieces = (e.lists > 1 ? e.D : row) / VEC;   // of 16 bytes: 8, 16 or 32, or a whole row's
    const int side = pieces < kWave ? idiv(kWave, pieces) : 1, my = idiv(lane, min(pieces, kWave)), first = lane - my * min(pieces, kWave);   // moves side by side
    for (int m = 0; m < n; m += 4 * side)
        for (int c0 = 0; c0 < pieces; c0 += kWave) {
            const int c = c0 + first;
            u32x4 k[4], v[4];
            int64_t ys[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = m + u * side + my;
                const int64_t xs = __shfl(x, min(i, kWave - 1));
                ys[u] = __shfl(y, min(i, kWave - 1));
                if (i >= n || my >= side || c >= pieces) ys[u] = -1;
                if (ys[u] >= 0) {
                    k[u] = ld16(Kp + xs + c * VEC);
                    v[u] = ld16(Vp + xs + c * VEC);
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (ys[u] >= 0) {
                    __builtin_nontemporal_store(k[u], reinterpret_cast<u32x4*>(Kp + ys[u] + c * VEC));
                    __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4*>(Vp + ys[u] + c * VEC));
                }
        }
}

// exclusive prefix sum over the 16 waves' values (uniform in a wave) and the total, from LDS
__device__ __forceinline__ uint32_t evict_before(const uint32_t* sums, int wave, uint32_t* total)
{
    const int lane = lane_id();
    const uint32_t w = sums[lane & 15];
    *total = wave_uniform((int)row16_sum_u32(w));
    return wave_uniform((int)row16_sum_u32((lane & 15) < wave ? w : 0u));
}

struct EvictShared {
    __attribute__((aligned(16))) uint32_t hist[kEvBins];
    uint32_t sumA[2][kEvWaves], sumB[2][kEvWaves];
    uint32_t key[kEvMembers], n_members;
    int32_t slot[kEvMembers];
    uint32_t bin[3];
    int32_t from[kEvFused], to[kEvFused];
    uint32_t last;
};

// weights and positions of four slots from j on (a list need not begin on 16 bytes); what lies behind the list is zero
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4u __attribute__((ext_vector_type(4), aligned(4)));
struct EvictRaw {
    f32x4 w;
    i32x4u p;
    __device__ __forceinline__ void load(const float* weights, const int32_t* pos, int j, int cap)
    {
        if (j + 4 <= cap) {
            w = *reinterpret_cast<const f32x4u*>(weights + j);
            p = *reinterpret_cast<const i32x4u*>(pos + j);
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) { w[u] = j + u < cap ? weights[j + u] : 0.f; p[u] = j + u < cap ? pos[j + u] : 0; }
        }
    }
    __device__ __forceinline__ void keys(uint32_t (&k)[4], int32_t n_sink, int64_t recent_from) const
    {
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = evict_key(w[u], p[u], n_sink, recent_from);
    }
};

// Counts of a bin in LDS; lanes with the first one's bin count together: weights that are all alike would queue up at one address.
__device__ __forceinline__ void evict_count(uint32_t* hist, uint32_t bin, bool on)
{
    const uint64_t act = __ballot(on);
    if (!act) return;
    const int lane = lane_id(), first = __ffsll((unsigned long long)act) - 1;
    const bool same = on && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, first);
    const uint32_t n = (uint32_t)__popcll(__ballot(same));
    if (on && (!same || lane == first)) atomicAdd(&hist[bin], same ? n : 1u);
}

// Of the 4096 bins, of which this thread holds h = those from 4 (1023 - t) on: the one that the `need`-th largest is in, how many of
// its members are needed and how many it has, left in sh.bin (two barriers inside, the second one behind the result).
__device__ __forceinline__ void evict_bin(EvictShared& sh, const u32x4& h, uint32_t need)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_uniform(tid >> 6);
    const uint32_t four = h.x + h.y + h.z + h.w, upto = wave_incl_scan(four);
    if (lane == kWave - 1) sh.sumA[0][wave] = upto;
    __syncthreads();
    uint32_t total, above = evict_before(sh.sumA[0], wave, &total) + upto - four;
    if (above < need && need <= above + four) {
        int u = 3;
        for (; need > above + h[u]; --u) above += h[u];
        sh.bin[0] = 4u * (uint32_t)(kEvThreads - 1 - tid) + (uint32_t)u;
        sh.bin[1] = need - above;
        sh.bin[2] = h[u];
    }
    __syncthreads();
}

// The need-th of n <= kEvMembers members in sh.key, sh.slot by rank, left in sh.bin[0], sh.bin[1]: four threads for each
__device__ __forceinline__ void evict_rank(EvictShared& sh, int n, uint32_t need)
{
    const int i = threadIdx.x >> 2, part = threadIdx.x & 3;
    uint32_t before = 0;
    if (i < n)
        for (int o = part; o < n; o += 4) before += sh.key[o] > sh.key[i] || (sh.key[o] == sh.key[i] && sh.slot[o] < sh.slot[i]);
    before += (uint32_t)__shfl_xor((int)before, 1);
    before += (uint32_t)__shfl_xor((int)before, 2);
    if (i < n && part == 0 && before == need - 1) { sh.bin[0] = sh.key[i]; sh.bin[1] = (uint32_t)sh.slot[i]; }
}

// One list by the calling workgroup.  NC: steps of a wave in registers, 0: any number, read anew (then e.fused must be 0)
template <typename T, int NC>
__device__ __forceinline__ void evict_select(EvictShared& sh, const PagedCache& a, const EvictArgs& e, T* Kp, T* Vp, int32_t* seq_len, int rowi)
{
    constexpr int NR = NC > 0 ? NC : 4;
    const int b = idiv(rowi, e.lists), tid = threadIdx.x, lane = tid & 63, wave = wave_uniform(tid >> 6);
    const float* w = e.weights + (size_t)rowi * a.cap;
    const int32_t* p = e.pos + (size_t)rowi * a.cap;
    const int steps = (a.cap + kEvChunk - 1) / kEvChunk, slot0 = wave * steps * kEvStep + lane * 4;
    // requested with the length; what lies behind it is dropped later
    EvictRaw raw[NR];
    if constexpr (NC > 0) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (c < steps) raw[c].load(w, p, slot0 + c * kEvStep, a.cap);
    }
    const int S = min(max(seq_len[b], 0), a.cap);
    const int64_t recent_from = (int64_t)e.q_pos[b] - e.n_recent;
    int32_t* src = e.src ? e.src + (size_t)rowi * e.n_keep : nullptr;
    if (S <= e.n_keep) {
        if (src)
            for (int j = tid; j < e.n_keep; j += kEvThreads) src[j] = j < S ? j : -1;
        if (tid == 0 && !e.fused) e.moves[rowi] = -1;
        // (nobody counts on this list's arrival: the others of the sequence end here too)
        return;
    }
    uint32_t kr[NR][4];
    if constexpr (NC > 0) {
#pragma unroll
        for (int c = 0; c < NC; ++c) raw[c].keys(kr[c], e.n_sink, recent_from);
    }
    // f(step, first slot of this lane, its four keys), in the order of the slots
    auto visit = [&](auto f) {
        if constexpr (NC > 0) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (c < steps) f(c, slot0 + c * kEvStep, kr[c]);   // uniform
        } else {
            for (int c0 = 0; c0 < steps && slot0 - lane * 4 + c0 * kEvStep < S; c0 += NR) {
                EvictRaw r[NR];
#pragma unroll
                for (int c = 0; c < NR; ++c)
                    if (c0 + c < steps) r[c].load(w, p, slot0 + (c0 + c) * kEvStep, a.cap);
#pragma unroll
                for (int c = 0; c < NR; ++c)
                    if (c0 + c < steps) {
                        uint32_t k[4];
                        r[c].keys(k, e.n_sink, recent_from);
                        f(c0 + c, slot0 + (c0 + c) * kEvStep, k);
                    }
            }
        }
    };

    int32_t* const from = e.fused ? sh.from : e.from + (size_t)rowi * e.move_cap;
    int32_t* const to = e.fused ? sh.to : e.to + (size_t)rowi * e.move_cap;
    auto make_moves = [&](int n) {   // every wave some of them
        const int each = (n + kEvWaves - 1) / kEvWaves, m0 = wave * each, mine = min(each, n - m0);
        if (mine > 0) evict_move<T>(a, e, Kp, Vp, rowi, sh.from + m0, sh.to + m0, mine);
    };
    auto done = [&](int left) {      // moves that are left to the second launch; without one, the last of the sequence's lists sets the length
        if (tid != 0) return;
        if (!e.fused) e.moves[rowi] = left;
        else if (e.lists == 1 || arrive(e.count + b, (uint32_t)e.lists) == (uint32_t)e.lists - 1) seq_len[b] = e.n_keep;
    };

    // ---- few leave: the lowest, one by one ----
    if constexpr (NC > 0)
        if (S - e.n_keep <= kEvFew) {
            const int n_out = S - e.n_keep;
            if (src)
                for (int j = tid; j < e.n_keep; j += kEvThreads) src[j] = j;   // (the moves' are written behind them)
            uint32_t last = 0;
            int last_slot = 0x7fffffff, out = -1;   // lane i: the slot that left in round i
            for (int r = 0; r < n_out; ++r) {
                uint32_t low = 0xffffffffu;
                int at = -1;
                visit([&](int, int j0, const uint32_t (&k)[4]) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int j = j0 + u;
                        if (j < S && (k[u] > last || (k[u] == last && j < last_slot)) && (k[u] < low || (k[u] == low && j > at))) { low = k[u]; at = j; }
                    }
                });
                const uint32_t wl = wave_min_u32(low);
                const uint32_t ws = wave_max_u32(low == wl ? (uint32_t)(at + 1) : 0u);
                if (lane == 0) { sh.sumA[r & 1][wave] = wl; sh.sumB[r & 1][wave] = ws; }
                __syncthreads();
                const uint32_t al = sh.sumA[r & 1][lane & 15], as = sh.sumB[r & 1][lane & 15];
                last = wave_min_u32(al);
                last_slot = (int)wave_max_u32(al == last ? as : 0u) - 1;
                if (lane == r) out = last_slot;
            }
            const bool left = lane < n_out, fr = left && out < e.n_keep;
            bool late = left;            // slot n_keep + lane, unless it is among those that left
            int rank = 0;
            for (int i = 0; i < n_out; ++i) {
                const int o = __builtin_amdgcn_readlane(out, i);
                rank += o < out;
                late = late && o != e.n_keep + lane;
            }
            const uint64_t late_of = __ballot(late);
            if (wave == 0) {
                if (fr) sh.to[rank] = out;
                if (late) sh.from[__popcll(late_of & ((1ull << lane) - 1))] = e.n_keep + lane;
            }
            __syncthreads();
            make_moves(__popcll(late_of));
            done(0);
            return;
        }

    // ---- threshold: what is above (key, slot) stays, as do that key's slots up to that slot ----
    uint32_t key = 0, need = (uint32_t)e.n_keep, members = (uint32_t)S;
    int slot = 0x7fffffff;
    for (int i = tid; i < kEvBins; i += kEvThreads) sh.hist[i] = 0;
    if (tid == 0) sh.n_members = 0;
    __syncthreads();
    for (int shift = 20, bits = 12;;) {
        visit([&](int, int j0, const uint32_t (&k)[4]) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                evict_count(sh.hist, k[u] >> shift & ((1u << bits) - 1), j0 + u < S && (shift == 20 || k[u] >> (shift + bits) == key));
        });
        __syncthreads();
        u32x4* const four = reinterpret_cast<u32x4*>(&sh.hist[4 * (kEvThreads - 1 - tid)]);
        const u32x4 h = *four;
        *four = u32x4{0u, 0u, 0u, 0u};
        evict_bin(sh, h, need);
        key = key << bits | sh.bin[0];
        need = sh.bin[1];
        members = sh.bin[2];
        if (need == members) { key = (key << shift) - 1u; slot = -1; break; }   // the bin stays whole (bin 0 cannot: then all would)
        if (members <= (uint32_t)kEvMembers || shift == 0) {
            const uint32_t bin_key = key;
            if (members <= (uint32_t)kEvMembers) {
                visit([&](int, int j0, const uint32_t (&k)[4]) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (j0 + u < S && k[u] >> shift == bin_key) {
                            const uint32_t i = atomicAdd(&sh.n_members, 1u);
                            sh.key[i] = k[u];
                            sh.slot[i] = j0 + u;
                        }
                });
                __syncthreads();
                evict_rank(sh, (int)members, need);
            } else {   // many slots of one key: the need-th of them
                uint32_t mine = 0;
                visit([&](int, int j0, const uint32_t (&k)[4]) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) mine += j0 + u < S && k[u] == bin_key;
                });
                mine = wave_sum_u32(mine);
                if (lane == 0) sh.sumB[0][wave] = mine;
                __syncthreads();
                uint32_t total, run = evict_before(sh.sumB[0], wave, &total);
                if (run < need && need <= run + mine)   // (one wave)
                    visit([&](int, int j0, const uint32_t (&k)[4]) {
                        uint32_t n = 0;
#pragma unroll
                        for (int u = 0; u < 4; ++u) n += j0 + u < S && k[u] == bin_key;
                        const uint32_t incl = wave_incl_scan(n);
                        uint32_t r = run + incl - n;
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (j0 + u < S && k[u] == bin_key && ++r == need) { sh.bin[0] = bin_key; sh.bin[1] = (uint32_t)(j0 + u); }
                        run += (uint32_t)__builtin_amdgcn_readlane((int)incl, kWave - 1);
                    });
            }
            __syncthreads();
            key = sh.bin[0];
            slot = (int)sh.bin[1];
            break;
        }
        if (shift == 20) shift = 8;
        else { shift = 0; bits = 8; }
    }

    // ---- the slots in order ----
    auto kinds = [&](int j0, const uint32_t (&k)[4], bool (&fr)[4], bool (&lt)[4]) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u;
            const bool kept = j < S && (k[u] > key || (k[u] == key && j <= slot));
            fr[u] = j < S && !kept && j < e.n_keep;
            lt[u] = kept && j >= e.n_keep;
            if (src && kept && j < e.n_keep) src[j] = j;
        }
    };
    uint32_t frees = 0, lates = 0;   // of the wave
    visit([&](int, int j0, const uint32_t (&k)[4]) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u;
            const bool kept = j < S && (k[u] > key || (k[u] == key && j <= slot));
            frees += (uint32_t)__popcll(__ballot(j < S && !kept && j < e.n_keep));
            lates += (uint32_t)__popcll(__ballot(kept && j >= e.n_keep));
        }
    });
    if (lane == 0) { sh.sumA[1][wave] = frees; sh.sumB[1][wave] = lates; }
    __syncthreads();
    uint32_t n_free, n_late;
    uint32_t f0 = evict_before(sh.sumA[1], wave, &n_free), l0 = evict_before(sh.sumB[1], wave, &n_late);
    visit([&](int, int j0, const uint32_t (&k)[4]) {
        bool fr[4], lt[4];
        kinds(j0, k, fr, lt);
        uint32_t n = 0;   // free, and moving in the upper half
#pragma unroll
        for (int u = 0; u < 4; ++u) n += fr[u] ? 1u : lt[u] ? 0x10000u : 0u;
        const uint32_t incl = wave_incl_scan(n), tot = (uint32_t)__builtin_amdgcn_readlane((int)incl, kWave - 1);
        uint32_t f = f0 + ((incl - n) & 0xffffu), l = l0 + ((incl - n) >> 16);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (fr[u]) to[f++] = j0 + u;
            if (lt[u]) from[l++] = j0 + u;
        }
        f0 += tot & 0xffffu;
        l0 += tot >> 16;
    });
    if (!e.fused) {
        done((int)n_free);
        return;
    }
    __syncthreads();
    make_moves((int)n_free);
    done(0);
}

// grid (B * lists)
template <typename T, int NC>
__global__ __launch_bounds__(kEvThreads) void paged_evict_select_kernel(PagedCache a, EvictArgs e, T* __restrict__ Kp, T* __restrict__ Vp, int32_t* seq_len)
{
    __shared__ EvictShared sh;
    evict_select<T, NC>(sh, a, e, Kp, Vp, seq_len, blockIdx.x);
}

// ---- longer tables: a workgroup for each 4096 slots, in three launches (a list's keys are too many instructions for one compute unit:
// 4 x (82 000 of 4 lists) 47 us in one workgroup each) ----
// hist     the chunks' histograms of the leading 12 bits added up for the list; the last chunk to arrive finds the bin
// (split   tables of more than 131072 slots: the same with the next 12 bits, if the bin has more members than a workgroup ranks)
// members  every chunk counts what is certain to become free or to move, and lists the bin's members; the last one ranks them and
//          leaves the threshold and the chunks' places in the lists of moves.  A list with more members than that (one weight many times
//          over, or a bin that holds many: uniform weights in 65536 slots) is done by that workgroup alone.
// emit     every chunk writes its part of the lists of moves
constexpr int kEvCand = 4096;
constexpr int kEvMaxChunks = (1 << 20) / kEvChunk;
enum { kEvKey = 0, kEvNeed, kEvCount, kEvShift, kEvSlot, kEvDone, kEvState = 8 };   // a list's state

struct EvictChain {
    uint32_t *hist, *n_cand, *arrived;   // [rows][kEvBins], [rows], [rows]: zero between launches
    uint32_t* state;                     // [rows][kEvState]
    uint2* cand;                         // [rows][kEvCand]: key, slot
    uint2* part;                         // [rows][chunks]: free and moving slots of a chunk, then the places of its first ones
    int chunks;                          // of a list's capacity
};

__device__ __forceinline__ uint32_t ldu_device(const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint2 ldu2_device(const uint2* p)
{
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_uint2((uint32_t)v, (uint32_t)(v >> 32));
}
__device__ __forceinline__ void stu2_device(uint2* p, uint32_t x, uint32_t y)
{
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), (uint64_t)y << 32 | x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// the calling chunk of a list: its keys, four for each thread
struct EvictPiece {
    int b, S, j0;
    uint32_t k[4];
    __device__ __forceinline__ EvictPiece(const PagedCache& a, const EvictArgs& e, const int32_t* seq_len, int rowi, int chunk)
    {
        b = idiv(rowi, e.lists);
        j0 = chunk * kEvChunk + 4 * threadIdx.x;
        EvictRaw r;
        r.load(e.weights + (size_t)rowi * a.cap, e.pos + (size_t)rowi * a.cap, j0, a.cap);
        S = min(max(seq_len[b], 0), a.cap);
        r.keys(k, e.n_sink, (int64_t)e.q_pos[b] - e.n_recent);
    }
    __device__ __forceinline__ int live() const { return (S + kEvChunk - 1) / kEvChunk; }   // chunks that hold slots in use
};

// is this the last of the list's `n` chunks to arrive?  (for all threads; stores and atomics before are the device's by then)
__device__ __forceinline__ bool evict_last(EvictShared& sh, uint32_t* count, int n)
{
    device_stores_done();
    __syncthreads();
    if (threadIdx.x == 0) sh.last = arrive(count, (uint32_t)n) == (uint32_t)n - 1;
    __syncthreads();
    return sh.last != 0;
}

// grid (chunks, rows)
__global__ __launch_bounds__(kEvThreads) void paged_evict_hist_kernel(PagedCache a, EvictArgs e, EvictChain c, const int32_t* __restrict__ seq_len, int split)
{
    __shared__ EvictShared sh;
    const int rowi = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x;
    uint32_t* const st = c.state + (size_t)rowi * kEvState;
    const uint32_t prefix = split ? st[kEvKey] : 0u;
    if (split && st[kEvCount] <= (uint32_t)kEvCand) return;
    EvictPiece x(a, e, seq_len, rowi, chunk);
    if (x.S <= e.n_keep) {
        int32_t* src = e.src ? e.src + (size_t)rowi * e.n_keep : nullptr;
        if (src && !split)
            for (int j = chunk * kEvChunk + tid; j < min(e.n_keep, (chunk + 1) * kEvChunk); j += kEvThreads) src[j] = j < x.S ? j : -1;
        if (tid == 0 && chunk == 0) { e.moves[rowi] = -1; st[kEvCount] = 0; st[kEvDone] = 1; }
        return;
    }
    if (chunk >= x.live()) return;
    u32x4* const four = reinterpret_cast<u32x4*>(&sh.hist[4 * (kEvThreads - 1 - tid)]);
    *four = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) evict_count(sh.hist, split ? x.k[u] >> 8 & 0xfffu : x.k[u] >> 20, x.j0 + u < x.S && (!split || x.k[u] >> 20 == prefix));
    __syncthreads();
    uint32_t* const g = c.hist + (size_t)rowi * kEvBins + 4 * (kEvThreads - 1 - tid);
    const u32x4 h = *four;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (h[u]) atomicAdd(g + u, h[u]);
    if (!evict_last(sh, c.arrived + rowi, x.live())) return;
    u32x4 all;
#pragma unroll
    for (int u = 0; u < 4; ++u) { all[u] = ldu_device(g + u); g[u] = 0u; }
    evict_bin(sh, all, split ? st[kEvNeed] : (uint32_t)e.n_keep);
    if (tid == 0) {
        st[kEvKey] = split ? prefix << 12 | sh.bin[0] : sh.bin[0];
        st[kEvNeed] = sh.bin[1];
        st[kEvCount] = sh.bin[2];
        st[kEvShift] = split ? 8u : 20u;
        st[kEvDone] = 0u;
    }
}

// grid (chunks, rows)
template <typename T>
__global__ __launch_bounds__(kEvThreads) void paged_evict_members_kernel(PagedCache a, EvictArgs e, EvictChain c, T* __restrict__ Kp, T* __restrict__ Vp,
                                                                        int32_t* seq_len)
{
    __shared__ EvictShared sh;
    __shared__ uint32_t sFree[kEvMaxChunks], sLate[kEvMaxChunks];
    const int rowi = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = wave_uniform(tid >> 6);
    uint32_t* const st = c.state + (size_t)rowi * kEvState;
    uint2* const cand = c.cand + (size_t)rowi * kEvCand;
    uint2* const part = c.part + (size_t)rowi * c.chunks;
    const uint32_t done = st[kEvDone], bin = st[kEvKey], shift = st[kEvShift], need0 = st[kEvNeed], members = st[kEvCount];
    EvictPiece x(a, e, seq_len, rowi, chunk);
    if (done || chunk >= x.live()) return;
    const bool whole = need0 == members, few = members <= (uint32_t)kEvCand;   // the bin stays whole; its members can be ranked
    if (!whole && !few) {
        if (chunk == 0) {
            evict_select<T, 0>(sh, a, e, Kp, Vp, seq_len, rowi);
            if (tid == 0) st[kEvDone] = 1u;
        }
        return;
    }
    uint32_t frees = 0, lates = 0, opens = 0, mine = 0;   // of the wave; bit u: this lane's slot u is a member
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int j = x.j0 + u;
        const uint32_t at = x.k[u] >> shift;
        const bool in = j < x.S, open = in && at == bin && !whole, kept = in && (whole ? at >= bin : at > bin);
        frees += (uint32_t)__popcll(__ballot(in && !open && !kept && j < e.n_keep));
        lates += (uint32_t)__popcll(__ballot(kept && j >= e.n_keep));
        opens += (uint32_t)__popcll(__ballot(open));
        mine |= (uint32_t)open << u;
    }
    if (lane == 0) { sh.sumA[0][wave] = frees; sh.sumB[0][wave] = lates; sh.sumA[1][wave] = opens; }
    __syncthreads();
    uint32_t n_open;
    uint32_t at_open = evict_before(sh.sumA[1], wave, &n_open);
    if (tid == 0 && n_open) sh.last = atomicAdd(c.n_cand + rowi, n_open);   // the chunk's members take consecutive places
    if (wave == 1) {
        const uint32_t f = row16_sum_u32(sh.sumA[0][lane & 15]), l = row16_sum_u32(sh.sumB[0][lane & 15]);
        if (lane == 0) stu2_device(part + chunk, f, l);
    }
    if (n_open) {   // uniform
        __syncthreads();
        const uint32_t n = (uint32_t)__popc(mine), incl = wave_incl_scan(n);
        uint32_t to = sh.last + at_open + incl - n;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (mine >> u & 1) stu2_device(cand + to++, x.k[u], (uint32_t)(x.j0 + u));
    }
    const int n_chunks = x.live();
    if (!evict_last(sh, c.arrived + rowi, n_chunks)) return;
    if (tid == 0) c.n_cand[rowi] = 0u;
    uint32_t f = 0, l = 0;
    if (tid < n_chunks) {
        const uint2 v = ldu2_device(part + tid);
        f = v.x; l = v.y;
    }
    uint32_t key = (bin << shift) - 1u;   // the whole bin: what is above this
    int slot = -1;
    uint2 m[kEvCand / kEvThreads];
    bool on[kEvCand / kEvThreads];
#pragma unroll
    for (int i = 0; i < kEvCand / kEvThreads; ++i) {
        on[i] = !whole && (uint32_t)(tid + i * kEvThreads) < members;
        m[i] = on[i] ? ldu2_device(cand + tid + i * kEvThreads) : make_uint2(0u, 0u);
    }
    if (!whole) {
        uint32_t need = need0, n = members, prefix = bin, sft = shift;
        bool settled = false;
        for (int i = tid; i < kEvBins; i += kEvThreads) sh.hist[i] = 0;
        if (tid == 0) sh.n_members = 0;
        __syncthreads();
        while (n > (uint32_t)kEvMembers && sft > 0) {   // the next 12 bits, the last 8
            const uint32_t bits = min(12u, sft);
            sft -= bits;
#pragma unroll
            for (int i = 0; i < kEvCand / kEvThreads; ++i)
                evict_count(sh.hist, m[i].x >> sft & ((1u << bits) - 1), on[i] && m[i].x >> (sft + bits) == prefix);
            __syncthreads();
            u32x4* const four = reinterpret_cast<u32x4*>(&sh.hist[4 * (kEvThreads - 1 - tid)]);
            const u32x4 h = *four;
            *four = u32x4{0u, 0u, 0u, 0u};
            evict_bin(sh, h, need);
            prefix = prefix << bits | sh.bin[0];
            need = sh.bin[1];
            n = sh.bin[2];
            if (need == n) { key = (prefix << sft) - 1u; slot = -1; settled = true; break; }
            __syncthreads();   // (sh.bin is written again)
        }
        if (!settled && n <= (uint32_t)kEvMembers) {
#pragma unroll
            for (int i = 0; i < kEvCand / kEvThreads; ++i)
                if (on[i] && m[i].x >> sft == prefix) {
                    const uint32_t at = atomicAdd(&sh.n_members, 1u);
                    sh.key[at] = m[i].x;
                    sh.slot[at] = (int32_t)m[i].y;
                }
            __syncthreads();
            evict_rank(sh, (int)n, need);
            __syncthreads();
            key = sh.bin[0];
            slot = (int)sh.bin[1];
        } else if (!settled) {   // one key, many slots, in no order: the need-th of them by halving
            int lo = 0, hi = x.S - 1;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                uint32_t below = 0;
#pragma unroll
                for (int i = 0; i < kEvCand / kEvThreads; ++i) below += (uint32_t)__popcll(__ballot(on[i] && m[i].x == prefix && (int)m[i].y <= mid));
                __syncthreads();
                if (lane == 0) sh.sumA[0][wave] = below;
                __syncthreads();
                if (wave_uniform((int)row16_sum_u32(sh.sumA[0][lane & 15])) >= (int)need) hi = mid;
                else lo = mid + 1;
            }
            key = prefix;
            slot = lo;
        }
    }
    // the members' slots join what is certain
    if (tid < kEvMaxChunks) { sFree[tid] = f; sLate[tid] = l; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEvCand / kEvThreads; ++i)
        if (on[i]) {
            const int j = (int)m[i].y;
            const bool kept = m[i].x > key || (m[i].x == key && j <= slot);
            if (!kept && j < e.n_keep) atomicAdd(&sFree[j / kEvChunk], 1u);
            if (kept && j >= e.n_keep) atomicAdd(&sLate[j / kEvChunk], 1u);
        }
    __syncthreads();
    f = tid < n_chunks ? sFree[tid] : 0u;
    l = tid < n_chunks ? sLate[tid] : 0u;
    const uint32_t fu = wave_incl_scan(f), lu = wave_incl_scan(l);
    if (lane == kWave - 1) { sh.sumA[1][wave] = fu; sh.sumB[1][wave] = lu; }
    __syncthreads();
    uint32_t n_free, n_late;
    const uint32_t f0 = evict_before(sh.sumA[1], wave, &n_free) + fu - f, l0 = evict_before(sh.sumB[1], wave, &n_late) + lu - l;
    if (tid < n_chunks) part[tid] = make_uint2(f0, l0);
    if (tid == 0) { st[kEvKey] = key; st[kEvSlot] = (uint32_t)slot; e.moves[rowi] = (int32_t)n_free; }
}

// grid (chunks, rows)
__global__ __launch_bounds__(kEvThreads) void paged_evict_emit_kernel(PagedCache a, EvictArgs e, EvictChain c, const int32_t* __restrict__ seq_len)
{
    __shared__ uint32_t sums[kEvWaves];
    const int rowi = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = wave_uniform(tid >> 6);
    const uint32_t* const st = c.state + (size_t)rowi * kEvState;
    const uint32_t done = st[kEvDone], key = st[kEvKey];
    const int slot = (int)st[kEvSlot];
    const uint2 place = c.part[(size_t)rowi * c.chunks + chunk];
    EvictPiece x(a, e, seq_len, rowi, chunk);
    if (done || chunk >= x.live()) return;
    int32_t* src = e.src ? e.src + (size_t)rowi * e.n_keep : nullptr;
    bool fr[4], lt[4];
    uint32_t n = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int j = x.j0 + u;
        const bool kept = j < x.S && (x.k[u] > key || (x.k[u] == key && j <= slot));
        fr[u] = j < x.S && !kept && j < e.n_keep;
        lt[u] = kept && j >= e.n_keep;
        if (src && kept && j < e.n_keep) src[j] = j;
        n += fr[u] ? 1u : lt[u] ? 0x10000u : 0u;   // (no more than 4096 of either)
    }
    const uint32_t incl = wave_incl_scan(n);
    if (lane == kWave - 1) sums[wave] = incl;
    __syncthreads();
    uint32_t total;
    const uint32_t before = evict_before(sums, wave, &total) + incl - n;
    uint32_t f = place.x + (before & 0xffffu), l = place.y + (before >> 16);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (fr[u]) e.to[(size_t)rowi * e.move_cap + f++] = x.j0 + u;
        if (lt[u]) e.from[(size_t)rowi * e.move_cap + l++] = x.j0 + u;
    }
}

// grid (x, rows): the moves, `batch` of them a wave at a time; then the length
template <typename T>
__global__ __launch_bounds__(256) void paged_evict_move_kernel(PagedCache a, EvictArgs e, T* __restrict__ Kp, T* __restrict__ Vp, int32_t* seq_len, int batch)
{
    const int rowi = blockIdx.y, b = idiv(rowi, e.lists), wave = wave_uniform((int)threadIdx.x >> 6);
    const int n = e.moves[rowi];
    if (n < 0) return;
    if (blockIdx.x == 0 && rowi == b * e.lists && threadIdx.x == 0) seq_len[b] = e.n_keep;
    const int32_t *from = e.from + (size_t)rowi * e.move_cap, *to = e.to + (size_t)rowi * e.move_cap;
    for (int m = (blockIdx.x * 4 + wave) * batch; m < n; m += gridDim.x * 4 * batch) evict_move<T>(a, e, Kp, Vp, rowi, from + m, to + m, min(batch, n - m));
}

__global__ __launch_bounds__(256) void paged_clear_kernel(uint32_t* words, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) words[i] = 0u;
}

}  // namespace sals
