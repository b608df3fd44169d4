// C ABI of the paged key-value cache: descriptor validation, workspace carving and launches.  A source of its own, so that the
// code of the other kernels stays where it is; its place in the library is behind theirs.
#include "../../include/sals.h"

#include <algorithm>
#include <cmath>
#include <new>

#include "common.hpp"
#include "k_paged.hpp"

using namespace sals;

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline bool bad(const void* p) { return p == nullptr || (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline sals_status launch_status() { return hipGetLastError() == hipSuccess ? SALS_OK : SALS_ERR_HIP; }

struct PagedLayout {  // byte offsets into the workspace
    size_t count, sum, stat, final_stat, logits, moves, from, to, hist, n_cand, arrived, state, cand, part, total;
    size_t n_zero;   // words from `count` on that are zero between launches
    int chunks, tiles, groups, rows, lds, move_cap, logit_stride;   // of the attention: head tiles, workgroups, query heads of one, LDS
};

inline int capacity(const sals_paged_desc& d) { return d.max_pages * d.page_size; }

sals_status validate(const sals_paged_desc* d)
{
    if (!d) return SALS_ERR_INVALID_ARG;
    if (d->dtype != SALS_F32 && d->dtype != SALS_BF16) return SALS_ERR_INVALID_ARG;
    if (d->rope_style != SALS_ROPE_HALF && d->rope_style != SALS_ROPE_INTERLEAVED) return SALS_ERR_INVALID_ARG;
    if (!(d->rope_theta > 0.f) || !std::isfinite(d->rope_theta)) return SALS_ERR_INVALID_ARG;
    if (d->B < 1 || d->H_q < 1 || d->H_kv < 1 || d->d < 2 || (d->d & 1) || d->H_q % d->H_kv != 0) return SALS_ERR_INVALID_ARG;
    if (d->page_size < 1 || d->max_pages < 1 || d->n_pages < 1) return SALS_ERR_INVALID_ARG;
    if (d->weight_heads != 0 && d->weight_heads != 1 && d->weight_heads != d->H_kv) return SALS_ERR_INVALID_ARG;
    // what the kernels cover
    if (d->d != 64 && d->d != 128) return SALS_ERR_UNSUPPORTED;
    if (d->B > 1024 || d->H_q > 1024 || d->page_size > 2048) return SALS_ERR_UNSUPPORTED;
    if ((int64_t)d->B * d->weight_heads > 65535) return SALS_ERR_UNSUPPORTED;
    if ((int64_t)d->max_pages * d->page_size > (1 << 20)) return SALS_ERR_UNSUPPORTED;
    const int64_t page = (int64_t)d->page_size * d->H_kv * d->d, vec = d->dtype == SALS_BF16 ? 8 : 4;
    if (d->page_stride != 0 && (d->page_stride < page || d->page_stride % vec != 0)) return SALS_ERR_INVALID_ARG;
    if (d->page_stride > ((int64_t)1 << 55) / d->n_pages) return SALS_ERR_UNSUPPORTED;   // offsets are 64-bit bytes
    return SALS_OK;
}

PagedLayout make_layout(const sals_paged_desc& d)
{
    PagedLayout L{};
    const size_t H = (size_t)d.B * d.H_q, cap = (size_t)capacity(d);
    const int group = d.H_q / d.H_kv, tiles = ceil_div(group, kPgHeads), single = d.H_kv * tiles;
    L.tiles = tiles;
    // the kernel takes one KV head for each workgroup or two, by the lengths: room for either
    int pieces = 0, factors = 0;   // of query heads
    for (int lg = 0; lg <= (tiles == 1 && d.H_kv % 2 == 0 ? 1 : 0); ++lg) {
        const int heads = single >> lg, shares = std::max(1, kPgGroups / heads);
        L.groups = std::max(L.groups, tiles > 1 ? ceil_div(shares * d.H_kv, 8) * 8 * tiles : shares * heads);
        pieces = std::max(pieces, (2 * shares * heads) << lg);
        factors = std::max(factors, shares << lg);
    }
    L.rows = std::min(group, kPgHeads);
    L.lds = 4 * L.rows * std::max(kPgWaves * (d.d + 4), factors);   // the waves' sums, or the factors of the pieces: up to 66 KB
    L.logit_stride = ceil_div((int)cap, 32) * 32;
    L.move_cap = (int)cap / 2 + 1;   // (no more than half of the slots can move below the others)
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t r = at; at += align_up(bytes); return r; };
    const size_t rows = (size_t)d.B * d.weight_heads;
    // Eviction in long tables, a workgroup for each chunk of 4096 slots: beyond 32768 slots, and beyond 16384 as long as there are fewer lists
    // than keep the compute units busy (32000 slots in use: 1 list 43 -> 28 us, 4 lists 49 -> 35, 64 lists 72 -> 74, 256 lists 191 -> 268;
    // 16000 slots: 32 and 30, 37 and 36).  By the table, as lengths are on the device: short sequences in long tables take this way too.
    L.chunks = (int)cap > 8 * kEvChunk || ((int)cap > 4 * kEvChunk && rows < 64) ? ceil_div((int)cap, kEvChunk) : 0;
    L.count = take((size_t)d.B * single * 4);
    if (rows && L.chunks) {
        L.n_cand = take(rows * 4);
        L.arrived = take(rows * 4);
        L.hist = take(rows * kEvBins * 4);
    }
    L.n_zero = at / 4;
    L.sum = take((size_t)pieces * L.rows * d.d * 4);
    L.stat = take((size_t)pieces * L.rows * 8);
    L.final_stat = take(H * 8);
    if (d.weight_heads) {
        L.logits = take(H * L.logit_stride * 4);
        L.moves = take(rows * 4);
        L.from = take(rows * L.move_cap * 4);
        L.to = take(rows * L.move_cap * 4);
        if (L.chunks) {
            L.state = take(rows * kEvState * 4);
            L.cand = take(rows * kEvCand * 8);
            L.part = take(rows * L.chunks * 8);
        }
    }
    L.total = at;
    return L;
}

}  // namespace

struct sals_paged {
    sals_paged_desc d;
    PagedLayout L;
    unsigned char* ws;
    double log2_theta;
    bool prepared;
};

namespace {

PagedCache cache_of(const sals_paged* c, const int32_t* table, const int32_t* seq_len)
{
    const sals_paged_desc& d = c->d;
    PagedCache a;
    a.table = table; a.seq_len = seq_len;
    a.page_stride = d.page_stride ? d.page_stride : (int64_t)d.page_size * d.H_kv * d.d;
    a.page_mul = (uint32_t)(((1u << 31) + (uint32_t)d.page_size - 1) / (uint32_t)d.page_size);
    a.page_size = d.page_size; a.max_pages = d.max_pages; a.n_pages = d.n_pages; a.cap = capacity(d);
    a.B = d.B; a.H_kv = d.H_kv; a.group = d.H_q / d.H_kv;
    return a;
}

template <typename T> T* at(const sals_paged* c, size_t off) { return reinterpret_cast<T*>(c->ws + off); }

template <typename T, int D>
sals_status launch_append(const sals_paged* c, const void* k_new, const void* v_new, const int32_t* q_pos, const int32_t* table, void* Kp, void* Vp,
                          int32_t* seq_len, const int32_t* n_new, int n_tok, int32_t* pos, float* weights, hipStream_t st)
{
    const sals_paged_desc& d = c->d;
    const int tok = (int)std::min<int64_t>(kAppTok, ((int64_t)d.B * n_tok + 767) / 768);
    const dim3 grid(ceil_div(n_tok, tok), d.B);
    hipLaunchKernelGGL((paged_append_kernel<T, D>), grid, dim3(256), 0, st, cache_of(c, table, seq_len), static_cast<const T*>(k_new),
                       static_cast<const T*>(v_new), q_pos, static_cast<T*>(Kp), static_cast<T*>(Vp), seq_len, at<uint32_t>(c, c->L.count), n_new, n_tok, tok,
                       pos, weights, d.weight_heads, c->log2_theta, d.rope_style);
    return launch_status();
}

template <typename T, int D> auto attend_kernel(const sals_paged* c)
{
    return c->d.page_size % (PgBlock<T>::TB / 4) == 0 ? paged_attend_kernel<T, D, true> : paged_attend_kernel<T, D, false>;
}
template <typename T, int D> sals_status allow_attend_lds(const sals_paged* c)
{
    // (of the kernel, not of the context: what the largest group takes, or logits that are kept)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(attend_kernel<T, D>(c)), hipFuncAttributeMaxDynamicSharedMemorySize,
                               std::max(kPgHeads * std::max(kPgWaves * (D + 4), 2 * kPgGroups), kPgWaves * kPgKept) * 4) == hipSuccess ? SALS_OK : SALS_ERR_HIP;
}

template <typename T, int D>
sals_status launch_attend(const sals_paged* c, const void* q, const int32_t* q_pos, const int32_t* table, const void* Kp, const void* Vp,
                          const int32_t* seq_len, float* weights, void* out, hipStream_t st)
{
    const sals_paged_desc& d = c->d;
    const PagedCache a = cache_of(c, table, seq_len);
    const PagedLayout& L = c->L;
    float* logits = weights ? at<float>(c, L.logits) : nullptr;
    const PagedParts parts{at<float>(c, L.sum), at<float2>(c, L.stat), at<uint32_t>(c, L.count), at<float2>(c, L.final_stat), L.rows};
    const float scale = (float)(1.4426950408889634074 / std::sqrt((double)D));
    // (64 KB of LDS for runs of logits: not where no wave can have more than two blocks, 0.5 us)
    const int keep = logits && (int64_t)d.B * ceil_div(a.cap, PgBlock<T>::TB) >= 16 * (kPgGroups / (d.H_kv * L.tiles)) ? 1 : 0;
    const int lds = keep ? std::max(L.lds, kPgWaves * kPgKept * 4) : L.lds;
    hipLaunchKernelGGL((attend_kernel<T, D>(c)), dim3(L.groups), dim3(kPgWaves * 64), lds, st, seq_len, d.B, a.cap, d.H_kv, L.tiles, a,
                       static_cast<const T*>(q), q_pos, static_cast<const T*>(Kp), static_cast<const T*>(Vp), static_cast<T*>(out), parts, logits,
                       L.logit_stride, keep, scale, c->log2_theta, d.rope_style);
    if (launch_status() != SALS_OK || !weights) return launch_status();
    hipLaunchKernelGGL(paged_weights_kernel, dim3(std::min(64, ceil_div(a.cap, 1024)), d.weight_heads, d.B), dim3(256), 0, st, a, logits,
                       at<float2>(c, L.final_stat), L.logit_stride, weights);
    return launch_status();
}

template <typename T>
sals_status launch_evict(const sals_paged* c, const int32_t* q_pos, const int32_t* table, void* Kp, void* Vp, int32_t* seq_len, int32_t* pos,
                         float* weights, int n_keep, int n_sink, int n_recent, int32_t* src, hipStream_t st)
{
    const sals_paged_desc& d = c->d;
    const PagedCache a = cache_of(c, table, seq_len);
    EvictArgs e;
    e.q_pos = q_pos; e.pos = pos; e.weights = weights; e.src = src;
    e.moves = at<int32_t>(c, c->L.moves); e.from = at<int32_t>(c, c->L.from); e.to = at<int32_t>(c, c->L.to);
    e.count = at<uint32_t>(c, c->L.count);
    e.lists = d.weight_heads; e.n_keep = n_keep; e.n_sink = n_sink; e.n_recent = n_recent; e.move_cap = c->L.move_cap; e.D = d.d;
    const int rows = d.B * d.weight_heads, most = std::min(n_keep, a.cap - n_keep);   // moves of a list
    e.fused = most <= kEvFused;
    T *const K = static_cast<T*>(Kp), *const V = static_cast<T*>(Vp);
    if (!c->L.chunks) {
        if (a.cap <= kEvChunk) hipLaunchKernelGGL((paged_evict_select_kernel<T, 1>), dim3(rows), dim3(kEvThreads), 0, st, a, e, K, V, seq_len);
        else if (a.cap > 2 * kEvChunk) hipLaunchKernelGGL((paged_evict_select_kernel<T, 8>), dim3(rows), dim3(kEvThreads), 0, st, a, e, K, V, seq_len);
        else hipLaunchKernelGGL((paged_evict_select_kernel<T, 2>), dim3(rows), dim3(kEvThreads), 0, st, a, e, K, V, seq_len);
    } else {
        e.fused = 0;
        const EvictChain ch{at<uint32_t>(c, c->L.hist), at<uint32_t>(c, c->L.n_cand), at<uint32_t>(c, c->L.arrived), at<uint32_t>(c, c->L.state),
                            at<uint2>(c, c->L.cand), at<uint2>(c, c->L.part), c->L.chunks};
        const dim3 grid(c->L.chunks, rows);
        hipLaunchKernelGGL(paged_evict_hist_kernel, grid, dim3(kEvThreads), 0, st, a, e, ch, seq_len, 0);
        if (launch_status() != SALS_OK) return SALS_ERR_HIP;
        if (a.cap > (1 << 17)) hipLaunchKernelGGL(paged_evict_hist_kernel, grid, dim3(kEvThreads), 0, st, a, e, ch, seq_len, 1);
        if (launch_status() != SALS_OK) return SALS_ERR_HIP;
        hipLaunchKernelGGL((paged_evict_members_kernel<T>), grid, dim3(kEvThreads), 0, st, a, e, ch, K, V, seq_len);
        if (launch_status() != SALS_OK) return SALS_ERR_HIP;
        hipLaunchKernelGGL(paged_evict_emit_kernel, grid, dim3(kEvThreads), 0, st, a, e, ch, seq_len);
    }
    if (launch_status() != SALS_OK || e.fused) return launch_status();
    // whole rows: four moves a wave, a head's part of them: eight (twice as many 2 % slower, four times 11 %)
    const int batch = e.lists == 1 && d.H_kv > 1 ? 4 : 8, x = std::max(1, std::min(ceil_div(4096, rows), ceil_div(most, 4 * batch)));
    hipLaunchKernelGGL((paged_evict_move_kernel<T>), dim3(x, rows), dim3(256), 0, st, a, e, K, V, seq_len, batch);
    return launch_status();
}

}  // namespace

extern "C" {

sals_status sals_paged_workspace_bytes(const sals_paged_desc* desc, size_t* bytes)
{
    if (!bytes) return SALS_ERR_INVALID_ARG;
    const sals_status s = validate(desc);
    if (s != SALS_OK) return s;
    *bytes = make_layout(*desc).total;
    return SALS_OK;
}

sals_status sals_paged_create(const sals_paged_desc* desc, void* d_workspace, size_t workspace_bytes, sals_paged** out)
{
    if (!out) return SALS_ERR_INVALID_ARG;
    *out = nullptr;
    const sals_status s = validate(desc);
    if (s != SALS_OK) return s;
    const PagedLayout L = make_layout(*desc);
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) % kAlign) != 0 || workspace_bytes < L.total) return SALS_ERR_WORKSPACE;
    sals_paged* c = new (std::nothrow) sals_paged;
    if (!c) return SALS_ERR_INVALID_ARG;
    c->d = *desc;
    c->L = L;
    c->ws = static_cast<unsigned char*>(d_workspace);
    c->log2_theta = std::log2((double)desc->rope_theta);
    c->prepared = false;
    *out = c;
    return SALS_OK;
}

void sals_paged_destroy(sals_paged* ctx) { delete ctx; }

#define SALS_PAGED(D_, CALL)                                                                     \
    (D_.dtype == SALS_BF16 ? (D_.d == 128 ? CALL(bf16_t, 128) : CALL(bf16_t, 64))               \
                           : (D_.d == 128 ? CALL(float, 128) : CALL(float, 64)))

sals_status sals_paged_prepare(sals_paged* ctx, void* hip_stream)
{
    if (!ctx) return SALS_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &cap) != hipSuccess) return SALS_ERR_HIP;
    if (cap != hipStreamCaptureStatusNone) return SALS_ERR_INVALID_ARG;
    hipLaunchKernelGGL(paged_clear_kernel, dim3((unsigned)std::min<size_t>(4096, (ctx->L.n_zero + 255) / 256)), dim3(256), 0, st, at<uint32_t>(ctx, ctx->L.count),
                       ctx->L.n_zero);
    if (launch_status() != SALS_OK || hipStreamSynchronize(st) != hipSuccess) return SALS_ERR_HIP;
#define SALS_CALL(T, D) allow_attend_lds<T, D>(ctx)
    if (SALS_PAGED(ctx->d, SALS_CALL) != SALS_OK) return SALS_ERR_HIP;
#undef SALS_CALL
    ctx->prepared = true;
    return SALS_OK;
}

sals_status sals_paged_append(sals_paged* ctx, const void* k_new, const void* v_new, const int32_t* q_pos, const int32_t* table, void* Kp, void* Vp,
                              int32_t* seq_len, const int32_t* n_new, int32_t n_tok, int32_t* pos, float* weights, void* hip_stream)
{
    if (!ctx || !ctx->prepared || bad(k_new) || bad(v_new) || !q_pos || !table || bad(Kp) || bad(Vp) || !seq_len) return SALS_ERR_INVALID_ARG;
    if (n_tok < 1 || n_tok > (1 << 20)) return SALS_ERR_INVALID_ARG;
    if (ctx->d.weight_heads ? bad(pos) || bad(weights) : pos || weights) return SALS_ERR_INVALID_ARG;
#define SALS_CALL(T, D) \
    launch_append<T, D>(ctx, k_new, v_new, q_pos, table, Kp, Vp, seq_len, n_new, n_tok, pos, weights, static_cast<hipStream_t>(hip_stream))
    return SALS_PAGED(ctx->d, SALS_CALL);
#undef SALS_CALL
}

sals_status sals_paged_attend(sals_paged* ctx, const void* q, const int32_t* q_pos, const int32_t* table, const void* Kp, const void* Vp,
                              const int32_t* seq_len, float* weights, void* out, void* hip_stream)
{
    if (!ctx || !ctx->prepared || bad(q) || !q_pos || !table || bad(Kp) || bad(Vp) || !seq_len || bad(out)) return SALS_ERR_INVALID_ARG;
    if (weights && (!ctx->d.weight_heads || bad(weights))) return SALS_ERR_INVALID_ARG;
#define SALS_CALL(T, D) launch_attend<T, D>(ctx, q, q_pos, table, Kp, Vp, seq_len, weights, out, static_cast<hipStream_t>(hip_stream))
    return SALS_PAGED(ctx->d, SALS_CALL);
#undef SALS_CALL
}

sals_status sals_paged_evict(sals_paged* ctx, const int32_t* q_pos, const int32_t* table, void* Kp, void* Vp, int32_t* seq_len, int32_t* pos,
                             float* weights, int32_t n_keep, int32_t n_sink, int32_t n_recent, int32_t* src, void* hip_stream)
{
    if (!ctx || !ctx->prepared || !q_pos || !table || bad(Kp) || bad(Vp) || !seq_len || bad(pos) || bad(weights)) return SALS_ERR_INVALID_ARG;
    if (!ctx->d.weight_heads || n_keep < 1 || n_keep > capacity(ctx->d) || n_sink < 0 || n_recent < 0) return SALS_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return ctx->d.dtype == SALS_BF16
               ? launch_evict<bf16_t>(ctx, q_pos, table, Kp, Vp, seq_len, pos, weights, n_keep, n_sink, n_recent, src, st)
               : launch_evict<float>(ctx, q_pos, table, Kp, Vp, seq_len, pos, weights, n_keep, n_sink, n_recent, src, st);
}

}  // extern "C"
