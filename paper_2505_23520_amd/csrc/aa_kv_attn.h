// What the kernels of kv_attn share.
#pragma once
#include "aa_kv.h"
#include "aa_kv_deal.h"

namespace aa {

struct AttnArgs {
    KvArgs a;
    const void* q;
    void* out;
    float *lse, *ws;
    int rows, tiles;                 // most rows of a KV head and sequence (N * grp), their row tiles
    int groups, whole;               // registers: work-groups that the line of units is dealt to; whole: a tile is one unit, however long
    int tell;                        // registers: the work-groups tell the joining kernel which tiles are shared
    int splits;                      // LDS: work-groups of a row tile
    float c;                         // sigma * log2 e
    float slack;                     // a reference is raised when a score exceeds it by this much: weights stay below 2^8
    FastDiv by_hkv, by_splits, by_grp, by_groups;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Table entries are read through the scalar cache: a load that the vector memory counter does not see.
using const_int = __attribute__((address_space(4))) const int;

// Keys that new token i of n of a sequence sees.
__device__ __forceinline__ int seen(const KvArgs& a, int len, int n, int i) {
    const long long room = (long long)a.max_pages << a.page_shift;
    long long x = a.causal ? (long long)len - n + i + 1 : len;
    if (x > room) x = room;
    return x < 0 ? 0 : (int)x;
}

// Keys of a share in the kernel through LDS (the last one's: what is left): every sequence's keys in as many shares, but no small ones.
__device__ __forceinline__ int share_keys(const AttnArgs& p, int len, int n) {
    const int all = seen(p.a, len, n, n - 1), keys = ((int)p.by_splits.div(all + p.splits - 1) + 127) & ~127;
    return keys < 256 ? 256 : keys;
}

// A work-group's rows and keys.  KV heads are dealt out first (to one XCD each where there are eight of them: its L2 then serves all row
// tiles of the head), the last rows, which see the most keys, before the others.
struct AttnPart {
    int b, hk, split, r0, rows, last, len, lo, hi, see_first;
    KvSeq sq;
};
template <int R> __device__ __forceinline__ bool attn_part(const AttnArgs& p, AttnPart& w) {
    const KvArgs& a = p.a;
    w.b = blockIdx.y;
    const unsigned rest = p.by_hkv.div(blockIdx.x), back = p.by_splits.div(rest);
    w.hk = (int)(blockIdx.x - rest * a.Hkv);
    w.split = (int)(rest - back * p.splits);
    w.r0 = (p.tiles - 1 - (int)back) * R;
    w.sq = kv_seq(a, w.b);
    w.len = a.kv_len[w.b];
    w.rows = w.sq.n * a.grp;
    if (w.r0 >= w.rows) return false;
    w.last = w.r0 + R < w.rows ? w.r0 + R - 1 : w.rows - 1;
    const int see_last = seen(a, w.len, w.sq.n, (int)p.by_grp.div(w.last));
    w.see_first = seen(a, w.len, w.sq.n, (int)p.by_grp.div(w.r0));
    const int keys = share_keys(p, w.len, w.sq.n);
    w.lo = w.split * keys;
    if (w.split && w.lo >= see_last) return false;
    w.hi = w.split == p.splits - 1 || see_last - w.lo < keys ? see_last : w.lo + keys;
    return true;
}

// Two bf16 values: the sign bits of those that are not finite; the finite ones alone.
__device__ __forceinline__ unsigned not_finite(unsigned x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ unsigned finite(unsigned x) { return x & ~((not_finite(x) >> 15) * 0xffffu); }

// Places of a row's results: its share in the workspace, its row maximum and sum there, its lse.
__device__ __forceinline__ long long share_of(const AttnArgs& p, const AttnPart& w, int row) {
    return (((long long)w.b * p.a.Hkv + w.hk) * p.rows + row) * p.splits + w.split;
}
__device__ __forceinline__ float* share_sums(const AttnArgs& p, int d) { return p.ws + (long long)p.a.B * p.a.Hkv * p.rows * p.splits * d; }
__device__ __forceinline__ long long lse_of(const KvArgs& a, const KvSeq& sq, int b, int h, int i) {
    return a.cu ? h * a.total + sq.row0 + i : ((long long)b * a.Hq + h) * a.N + i;
}

// Row tiles of 128 through LDS (d = 128, bf16 or 4-bit pages); hipError_t.
constexpr int kChunkRows = 128;
int launch_kv_chunk(const AttnArgs& p, int format, dim3 grid, hipStream_t st);

}  // namespace aa
