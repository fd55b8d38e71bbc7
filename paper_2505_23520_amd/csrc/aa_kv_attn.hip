// kv_attn: attention of new queries over the pages of the cache.
//
//   o_r = sum_j exp(s_rj - m_r) v_j / sum_j exp(s_rj - m_r),   s_rj = sigma <q_r, k_j>
//
// One pass over the keys with a running reference m and sum (online softmax), on the matrix cores.  The rows of a KV head's query
// heads and new tokens stand side by side (row r = token * grp + head): every key is read once for all of them.
//
// A wave takes 16 NT rows and a share of the keys and works alone until the end: no LDS and no barrier in the loop, K and V come from
// the pages straight into the registers that the matrix instruction reads.
//   S^T = K Q^T  (16x16: keys x rows).  A lane holds key lane % 16 of K, and 8 channels of each step at lane / 16 (=: g): 16 bytes of
//                a row as it lies.  Which channel stands where in the sum does not matter as long as Q has the same order.
//   O^T = V^T P^T (channels x rows).  The result of the first product is the second's right operand where it is: lane (row, g) holds
//                keys 4g .. 4g+3 of each half of the tile, and the sum over keys may run in that order too.  The left operand wants 8 keys of
//                one channel in a lane; a lane loads D/16 channels of each of its keys and two byte permutations turn four bf16 values.
// A lane's rows of S^T, O^T, m and the sum are all row lane % 16, so nothing crosses lanes unless a reference is raised.
#include <stdlib.h>
#include "aa_kv_attn.h"

namespace aa {
namespace {

using u32x2 = __attribute__((ext_vector_type(2))) unsigned;
using u32x4 = __attribute__((ext_vector_type(4))) unsigned;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;

constexpr int kWaves = 4;

enum { kRows32, kRows16, kRows4 };  // cached rows: float, bf16, 4 bits

template <int F> struct RowType { using type = __bf16; };
template <> struct RowType<kRows32> { using type = float; };

// One tile of keys in registers: TT halves of 16 keys, of which the first rows[h] exist and are seen by some row.
template <int F, int D> struct Tile;
template <int D> struct Tile<kRows16, D> {
    static constexpr int TT = 2, words = D / 32;
    u32x4 k[TT][D / 32];
    unsigned v[TT][4][words];
    int key, rows[TT];
};
template <int D> struct Tile<kRows4, D> {
    static constexpr int TT = 2, words = 1;
    unsigned k[TT][D / 32];
    unsigned v[TT][4][words];
    unsigned ks[TT], vs[TT];
    int key, rows[TT];
};
template <int D> struct Tile<kRows32, D> {
    static constexpr int TT = 1, words = D / 16;
    u32x4 k[TT][D / 16];
    unsigned v[TT][4][words];
    int key, rows[TT];
};

// What a wave needs to find a tile: its sequence's pages, the pools from its head on, and a lane's place in 16 keys (bytes).
struct Where {
    const_int* table;
    long long room;
    int shift, n_pages;
    const char *k, *v;
    const unsigned char *ks, *vs;
    long long k_page, v_page, k_row, v_row, ks_page, vs_page;
    int k_lane, v_lane[4], ks_lane, vs_lane, k_end, v_end;     // *_end: where the last row's bytes end, from the row's start
};

// The pages of a tile; -1: none.  Pages of 32 tokens and more hold both halves of one.
template <int TT> struct Pages { int p[TT]; };
template <int TT> __device__ __forceinline__ Pages<TT> pages_of(const Where& w, int key) {
    Pages<TT> x;
    x.p[0] = key < w.room ? w.table[key >> w.shift] : -1;
    if constexpr (TT == 2) {
        x.p[1] = x.p[0];
        if (__builtin_expect(w.shift == 4, 0)) x.p[1] = key + 16 < w.room ? w.table[(key >> 4) + 1] : -1;
    }
    return x;
}

// `bytes` bytes from x on, what is read behind them is 0.  Both are the same for the whole wave and said to be so: the compiler would
// otherwise take each load through a loop over the lanes' descriptors.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const void* x, int bytes) {
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)x), hi = __builtin_amdgcn_readfirstlane((unsigned)((uintptr_t)x >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)((uintptr_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
// n rows, `row` bytes apart, of which the last ends `end` bytes from its start.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const char* x, int n, long long row, int end) {
    const int bytes = n * (int)row - ((int)row - end);
    return bytes_at(x, n > 0 ? bytes : 0);
}

template <int N> __device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t rs, int at, unsigned* x) {
    static_assert(N == 1 || N == 2 || N % 4 == 0, "");
    if constexpr (N == 1) {
        x[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, at, 0, 0);
    } else if constexpr (N == 2) {
        const u32x2 u = __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0);
        x[0] = u[0]; x[1] = u[1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 u = __builtin_amdgcn_raw_buffer_load_b128(rs, at + 4 * i, 0, 0);
            x[i] = u[0]; x[i + 1] = u[1]; x[i + 2] = u[2]; x[i + 3] = u[3];
        }
    }
}

// Requests a tile, of which keys below hi count.  Rows that do not exist cost no memory traffic and come as zeros: a last tile's values behind
// the last key, whose weight is 0, may have any bits.
template <int F, int D>
__device__ __forceinline__ void load_tile(const Where& w, int key, int hi, const Pages<Tile<F, D>::TT>& pages, Tile<F, D>& t) {
    t.key = key;
    constexpr int TT = Tile<F, D>::TT;
    const char *k[TT], *v[TT];
    const unsigned char *ks[TT], *vs[TT];
#pragma unroll
    for (int h = 0; h < TT; ++h) {
        const bool there = (unsigned)pages.p[h] < (unsigned)w.n_pages;
        const int n = hi - (key + 16 * h);
        t.rows[h] = !there ? 0 : n < 16 ? n : 16;            // 0 and less: none
        if (h && __builtin_expect(w.shift > 4, 1)) {
            k[h] = k[0] + 16 * (int)w.k_row; v[h] = v[0] + 16 * (int)w.v_row;
            if constexpr (F == kRows4) { ks[h] = ks[0] + 16; vs[h] = vs[0] + 16; }
        } else {
            const long long pg = there ? pages.p[h] : 0;
            const int in = (key + 16 * h) & ((1 << w.shift) - 1);      // a page's rows span less than 2^31 bytes
            k[h] = w.k + pg * w.k_page + in * (int)w.k_row; v[h] = w.v + pg * w.v_page + in * (int)w.v_row;
            if constexpr (F == kRows4) { ks[h] = w.ks + pg * w.ks_page + in; vs[h] = w.vs + pg * w.vs_page + in; }
        }
    }
#pragma unroll
    for (int h = 0; h < TT; ++h) {
        const auto rs = rows_at(k[h], t.rows[h], w.k_row, w.k_end);
        if constexpr (F == kRows4) {
            load_words<D / 32>(rs, w.k_lane, t.k[h]);
            t.ks[h] = __builtin_amdgcn_raw_buffer_load_b8(bytes_at(ks[h], t.rows[h] > 0 ? 0x7fffffff : 0), w.ks_lane, 0, 0);
        } else {
#pragma unroll
            for (int s = 0; s < (F == kRows32 ? D / 16 : D / 32); ++s) t.k[h][s] = __builtin_amdgcn_raw_buffer_load_b128(rs, w.k_lane + 64 * s, 0, 0);
        }
    }
#pragma unroll
    for (int h = 0; h < TT; ++h) {
        const auto rs = rows_at(v[h], t.rows[h], w.v_row, w.v_end);
        if constexpr (F == kRows4)
            t.vs[h] = __builtin_amdgcn_raw_buffer_load_b32(bytes_at(vs[h], t.rows[h] > 0 ? 0x7fffffff : 0), w.vs_lane, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (F == kRows4 && D == 64) t.v[h][i][0] = (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rs, w.v_lane[i], 0, 0);
            else load_words<Tile<F, D>::words>(rs, w.v_lane[i], t.v[h][i]);
        }
    }
}

__device__ __forceinline__ unsigned fp4_pair(unsigned codes, float scale, int byte) {
    union { bf16x2 b; unsigned u; } r;
    switch (byte) {
        case 0: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0); break;
        case 1: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1); break;
        case 2: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2); break;
        default: r.b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3); break;
    }
    return r.u;
}

// State of a wave's rows: NT tiles of 16.
template <int F, int D, int NT> struct Rows {
    static constexpr int Q = F == kRows32 ? D / 16 : D / 32;
    u32x4 q[NT][Q];
    f32x4 o[NT][D / 16];
    float m[NT], l[NT];              // m: before the scale; l: this lane's keys alone
    int see[NT];                     // keys that the lane's row sees
};

template <int F, int D, int NT>
__device__ __forceinline__ void attend_tile(const AttnArgs& p, Tile<F, D>& t, int see_all, Rows<F, D, NT>& r) {
    constexpr int TT = Tile<F, D>::TT;
    const int g = (threadIdx.x & 63) >> 4;
    bool whole = true;
#pragma unroll
    for (int h = 0; h < TT; ++h) whole = whole && t.rows[h] == 16;
    if constexpr (F == kRows4) {
        if (!whole) {                // codes behind the last row are 0, their scales may be NaN
#pragma unroll
            for (int h = 0; h < TT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (4 * g + i >= t.rows[h]) t.vs[h] = (t.vs[h] & ~(255u << (8 * i))) | (127u << (8 * i));
        }
    }
    // scores
    f32x4 s[NT][TT];
    if constexpr (F == kRows32) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            s[n][0] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                union { u32x4 u; f32x4 f; } q, k;
                q.u = r.q[n][c];
                k.u = t.k[0][c];
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.f[e], q.f[e], s[n][0], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int h = 0; h < TT; ++h) {
            float scale = 0;
            if constexpr (F == kRows4) scale = __uint_as_float(t.ks[h] << 23);
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][h] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                union { u32x4 u; bf16x8 b; } k, q;
                if constexpr (F == kRows4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) k.u[e] = fp4_pair(t.k[h][c], scale, e);
                } else {
                    k.u = t.k[h][c];
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    q.u = r.q[n][c];
                    s[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.b, q.b, s[n][h], 0, 0, 0);
                }
            }
        }
    }
    // weights (scores and references before the scale c: one multiply-add makes the exponent of both)
    if (__builtin_expect(!(whole && t.key + 16 * TT <= see_all), 0)) {
        int base = 4 * g;
        asm volatile("" : "+v"(base));                   // else 50 instructions of this stand in every tile's way
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < TT; ++h) {
                const int left = r.see[n] - t.key - 16 * h, lim = left < t.rows[h] ? left : t.rows[h];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][h][i] = base + i < lim ? s[n][h][i] : -INFINITY;
            }
    }
    union { bf16x8 b; __bf16 e[8]; } pb[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float top = fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3]));
        if constexpr (TT == 2) top = fmaxf(top, fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3])));
        if (__builtin_expect(__any(top > r.m[n] + p.slack), 0)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m = fmaxf(top, r.m[n]);
            const float down = m == -INFINITY || m == r.m[n] ? 1.f : exp2f((r.m[n] - m) * p.c);
            r.m[n] = m;
            r.l[n] *= down;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) r.o[n][j] *= down;
        }
        const float ref = r.m[n] == -INFINITY ? 0.f : r.m[n] * p.c;
#pragma unroll
        for (int h = 0; h < TT; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][h][i] = __builtin_amdgcn_exp2f(fmaf(s[n][h][i], p.c, -ref));
                r.l[n] += s[n][h][i];
                if constexpr (F != kRows32) pb[n].e[4 * h + i] = (__bf16)s[n][h][i];
            }
    }
    // values
    if constexpr (F == kRows32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    r.o[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[0][i][j]), s[n][0][i], r.o[n][j], 0, 0, 0);
    } else {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {              // two channels at a time
            unsigned x[TT][4];
#pragma unroll
            for (int h = 0; h < TT; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (F == kRows4) x[h][i] = fp4_pair(t.v[h][i][0], __uint_as_float(((t.vs[h] >> (8 * i)) & 255u) << 23), c);
                    else x[h][i] = t.v[h][i][c];
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                union { u32x4 u; bf16x8 b; } v;
#pragma unroll
                for (int h = 0; h < TT; ++h)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        v.u[2 * h + i] = __builtin_amdgcn_perm(x[h][2 * i + 1], x[h][2 * i], e ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    r.o[n][2 * c + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.b, pb[n].b, r.o[n][2 * c + e], 0, 0, 0);
            }
        }
    }
}

template <int F, int D, int NT>
__global__ __launch_bounds__(64 * kWaves, NT == 1 ? 2 : 1) void kv_attn_kernel(AttnArgs p) {
    using T = typename RowType<F>::type;
    constexpr int item = sizeof(T), TT = Tile<F, D>::TT, TK = 16 * TT, R = 16 * NT, P = D + 4;
    __shared__ float s_o[kWaves][16][P];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const KvArgs& a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    AttnPart wp;
    const bool work = attn_part<R>(p, wp);
    const int b = wp.b, hk = wp.hk, r0 = wp.r0, rows = wp.rows, hi = wp.hi;
    const KvSeq sq = wp.sq;

    Where w;
    w.table = (const_int*)(a.table + b * a.table_stride);
    w.room = (long long)a.max_pages << a.page_shift;
    w.shift = a.page_shift;
    w.n_pages = a.n_pages;
    // tiles of the chunk go to the waves in turn (the first one's pages are on their way with the sequence's length)
    int key = wp.lo + wave * TK;
    Pages<TT> pages = pages_of<TT>(w, key);
    if (!work) return;
    constexpr int unit = F == kRows4 ? 1 : item, row_bytes = F == kRows4 ? D / 2 : D * item;
    w.k = a.kc + hk * a.kcs[1] * unit; w.v = a.vc + hk * a.vcs[1] * unit;
    w.k_page = a.kcs[0] * unit; w.v_page = a.vcs[0] * unit;
    w.k_row = a.kcs[2] * unit; w.v_row = a.vcs[2] * unit;
    w.k_end = w.v_end = row_bytes;
    w.k_lane = n16 * (int)w.k_row + g * (F == kRows4 ? D / 8 : 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) w.v_lane[i] = (4 * g + i) * (int)w.v_row + n16 * (row_bytes / 16);
    if constexpr (F == kRows4) {
        w.ks = a.ksc + hk * a.kss[1]; w.vs = a.vsc + hk * a.vss[1];
        w.ks_page = a.kss[0]; w.vs_page = a.vss[0];
        w.ks_lane = n16 + g * (D / 4) / kFp4Group * (int)a.kss[2];
        w.vs_lane = 4 * g + n16 * (D / 16) / kFp4Group * (int)a.vss[2];
    }
    Tile<F, D> t0, t1;
    load_tile<F, D>(w, key, hi, pages, t0);

    Rows<F, D, NT> r;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = r0 + 16 * n + n16 < rows ? r0 + 16 * n + n16 : rows - 1;
        const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
        r.see[n] = seen(a, wp.len, sq.n, i);
        r.m[n] = -INFINITY;
        r.l[n] = 0.f;
        const char* q = (const char*)p.q + kv_row(a, a.qs, b, sq.row0, i, h) * item;
#pragma unroll
        for (int c = 0; c < Rows<F, D, NT>::Q; ++c)
            r.q[n][c] = *(const u32x4*)(q + (F == kRows4 ? (D / 2) * g + 16 * c : 64 * c + 16 * g));
#pragma unroll
        for (int j = 0; j < D / 16; ++j) r.o[n][j] = f32x4{0, 0, 0, 0};
    }

    // Two tiles in registers, one loading while the other is attended.  Behind the last tile one without rows is loaded, so that every
    // path has as much in flight.
    if (key < hi) {
        pages = pages_of<TT>(w, key + kWaves * TK);
        for (;;) {
            key += kWaves * TK;
            load_tile<F, D>(w, key, hi, pages, t1);
            pages = pages_of<TT>(w, key + kWaves * TK);
            attend_tile<F, D, NT>(p, t0, wp.see_first, r);
            if (key >= hi) break;
            key += kWaves * TK;
            load_tile<F, D>(w, key, hi, pages, t0);
            pages = pages_of<TT>(w, key + kWaves * TK);
            attend_tile<F, D, NT>(p, t1, wp.see_first, r);
            if (key >= hi) break;
        }
    }

    // the waves' rows together, 16 at a time
    const int x = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * (D / 16);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float l = r.l[n];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (n) __syncthreads();
        if (g == 0) { s_m[wave][n16] = r.m[n] * p.c; s_l[wave][n16] = l; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) s_o[wave][n16][(D / 16) * (4 * g + i) + j] = r.o[n][j][i];
        __syncthreads();
        const int row = r0 + 16 * n + x;
        if (row >= rows) continue;
        float m = -INFINITY, sum = 0.f, acc[D / 16] = {};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) m = fmaxf(m, s_m[k][x]);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const float f = exp2f(s_m[k][x] - ref);
            sum += f * s_l[k][x];
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc[j] += f * s_o[k][x][c0 + j];
        }
        const int i = (int)p.by_grp.div(row), h = hk * a.grp + row - i * a.grp;
        if (p.splits > 1) {
            const long long at = share_of(p, wp, row);
            float* o = p.ws + at * D + c0;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] = acc[j];
            if (c0 == 0) {
                float* ml = share_sums(p, D) + at * 2;
                ml[0] = m; ml[1] = sum;
            }
        } else {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T* o = (T*)p.out + kv_row(a, a.os, b, sq.row0, i, h) + c0;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] = (T)(acc[j] * inv);
            if (p.lse && c0 == 0)
                p.lse[lse_of(a, sq, b, h, i)] =
                    sum == 0.f ? -INFINITY : m * kLn2 + logf(sum);
        }
    }
}

// The shares of a row together, a work-group a row: first their maxima and sums, a share a thread, which leave a weight for each;
// then D / 4 threads a share, 1024 / D shares at once, 16 bytes of a share's row a thread.
constexpr int kMaxSplits = 1024;
template <class T, int D>
__global__ __launch_bounds__(256) void kv_join_kernel(AttnArgs p) {
    constexpr int L = D / 4, S = 256 / L;
    __shared__ float s_w[kMaxSplits];
    __shared__ float s_m[4], s_l[4];
    __shared__ f32x4 s_o[S][L];
    const KvArgs& a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = blockIdx.y;
    const unsigned row = p.by_hkv.div(blockIdx.x), hk = blockIdx.x - row * a.Hkv;
    const KvSeq sq = kv_seq(a, b);
    const int i = (int)p.by_grp.div(row), h = (int)hk * a.grp + row - i * a.grp;
    if (i >= sq.n) return;
    // a share wrote this row if its keys begin before those that the row's tile of rows sees end; before those of the row is enough
    const int see = seen(a, a.kv_len[b], sq.n, i);
    int parts = (int)(((long long)see + p.chunk - 1) / p.chunk);
    parts = parts > p.splits ? p.splits : parts < 1 ? 1 : parts;
    const long long at = (((long long)b * a.Hkv + hk) * p.rows + row) * p.splits;
    const float* o = p.ws + at * D;
    const float* ml = share_sums(p, D) + at * 2;
    float m = -INFINITY;
    for (int s = threadIdx.x; s < parts; s += 256) m = fmaxf(m, ml[2 * s]);
#pragma unroll
    for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    for (int s = threadIdx.x; s < parts; s += 256) {
        const float f = exp2f(ml[2 * s] - ref);
        s_w[s] = f;
        l += f * ml[2 * s + 1];
    }
#pragma unroll
    for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
    if (lane == 0) s_l[wave] = l;
    __syncthreads();
    l = s_l[0] + s_l[1] + s_l[2] + s_l[3];
    const int c = threadIdx.x % L, s0 = threadIdx.x / L;
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll 8
    for (int s = s0; s < parts; s += S) acc += s_w[s] * *(const f32x4*)(o + (long long)s * D + 4 * c);
    s_o[s0][c] = acc;
    __syncthreads();
    if (threadIdx.x >= L) return;
#pragma unroll
    for (int s = 1; s < S; ++s) acc += s_o[s][c];
    T* out = (T*)p.out + kv_row(a, a.os, b, sq.row0, i, h) + 4 * c;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (T)(l == 0.f ? 0.f : acc[e] / l);
    if (p.lse && c == 0) p.lse[lse_of(a, sq, b, h, i)] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

// Rows of a work-group: 16 or 32 a wave's registers hold beside two tiles of d = 128; more go through LDS, 128 at a time, or 64 where d is
// less (float: 32, there is no such kernel).
int tile_rows(long long rows, int d, int dtype) {
    if (rows <= 16) return 16;
    if (rows <= 32 || (d == 128 && dtype == 0)) return 32;
    return d == 128 ? kChunkRows : 64;
}

template <int F, int D>
int run(const AttnArgs& p, int R, hipStream_t st) {
    using T = typename RowType<F>::type;
    const long long x = (long long)p.a.Hkv * p.tiles * p.splits, rows = (long long)p.a.Hkv * p.rows;
    if (x > 0x7fffffffll || (p.splits > 1 && rows > 0x7fffffffll)) return -1;
    const dim3 grid((unsigned)x, p.a.B), block(64 * kWaves);
    int e;
    if (R == 16) e = (int)launch_kernel(kv_attn_kernel<F, D, 1>, grid, block, 0, st, p);
    else if (R == 32) e = (int)launch_kernel(kv_attn_kernel<F, D, 2>, grid, block, 0, st, p);
    else if constexpr (D < 128) e = (int)launch_kernel(kv_attn_kernel<F, D, 4>, grid, block, 0, st, p);
    else e = launch_kv_chunk(p, F == kRows4, grid, st);
    if (e != (int)hipSuccess || p.splits == 1) return e;
    return (int)launch_kernel(kv_join_kernel<T, D>, dim3((unsigned)rows, p.a.B), dim3(256), 0, st, p);
}

}  // namespace

KvSplit kv_split(int B, int Hq, int Hkv, int N, int d, int dtype, long long longest) {
    const long long rows = (long long)N * (Hq / Hkv), R = tile_rows(rows, d, dtype), tiles = (rows + R - 1) / R;
    const long long groups = tiles * B * Hkv;
    static const long long TG = getenv("KV_TG") ? atoll(getenv("KV_TG")) : 1024, MC = getenv("KV_MC") ? atoll(getenv("KV_MC")) : 2048, LC = getenv("KV_LC") ? atoll(getenv("KV_LC")) : 256;
    long long splits = (TG + groups - 1) / groups;
    if (tiles == 1 && splits < (longest + MC - 1) / MC) splits = (longest + MC - 1) / MC;
    if (splits > (longest + LC - 1) / LC) splits = (longest + LC - 1) / LC;
    if (splits < 1) splits = 1;
    if (splits > kMaxSplits) splits = kMaxSplits;
    const long long chunk = ((longest + splits - 1) / splits + 127) / 128 * 128;
    splits = (longest + chunk - 1) / chunk;
    KvSplit s;
    s.splits = splits < 1 ? 1 : (int)splits;
    s.chunk = chunk < 128 ? 128 : (int)chunk;
    s.ws_bytes = s.splits == 1 ? 0 : (size_t)B * Hkv * rows * s.splits * (d + 2) * 4;
    return s;
}

int launch_kv_attn(const KvArgs& a, int dtype, int format, int d, const KvSplit& sp, const void* q, void* out, float* lse, float* ws,
                   hipStream_t st) {
    AttnArgs p;
    p.a = a;
    p.q = q; p.out = out; p.lse = lse; p.ws = ws;
    p.splits = sp.splits; p.chunk = sp.chunk;
    p.rows = a.N * a.grp;
    const int R = tile_rows(p.rows, d, dtype);
    p.tiles = (p.rows + R - 1) / R;
    p.c = a.sigma * kLog2e;
    p.slack = fminf(8.f / p.c, 3.402823466e38f);
    p.by_hkv.set(a.Hkv); p.by_splits.set(sp.splits); p.by_grp.set(a.grp);
    if (dtype == 0) return d == 32 ? run<kRows32, 32>(p, R, st) : d == 64 ? run<kRows32, 64>(p, R, st) : d == 128 ? run<kRows32, 128>(p, R, st) : -1;
    if (format) return d == 64 ? run<kRows4, 64>(p, R, st) : d == 128 ? run<kRows4, 128>(p, R, st) : -1;
    return d == 64 ? run<kRows16, 64>(p, R, st) : d == 128 ? run<kRows16, 128>(p, R, st) : -1;
}

}  // namespace aa
