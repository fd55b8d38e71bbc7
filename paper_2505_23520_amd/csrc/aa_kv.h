// Paged key / value cache: what its kernels and their host side share.  Layouts are those of include/anchor_attention.h.
#pragma once
#include "aa_common.h"
#include "aa_kv_fp4.h"

namespace aa {

// The call's description as the kernels take it (plain data, by value).
struct KvArgs {
    int B, Hq, Hkv, N, grp;
    int page_shift, n_pages, max_pages;
    int causal, rot, interleaved;
    float sigma;
    long long qs[3], ks[3], vs[3], os[3], kos[3];           // elements
    long long kcs[3], vcs[3];                               // plain: elements; 4 bits: bytes
    long long kss[3], vss[3];                               // bytes
    char *kc, *vc;
    unsigned char *ksc, *vsc;
    const int *table;
    long long table_stride;
    const int *kv_len;
    const int *cu;
    long long total;                                        // rows of the token axis (fixed length: B * N)
};

// The new tokens of sequence b: their count and the row of the first.
struct KvSeq { int n; long long row0; };
__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int b) {
    KvSeq s;
    if (!a.cu) { s.n = a.N; s.row0 = (long long)b * a.N; return s; }
    const long long lo = a.cu[b], hi = a.cu[b + 1];
    s.row0 = lo;
    s.n = lo < 0 || hi > a.total || hi <= lo ? 0 : (int)(hi - lo < a.N ? hi - lo : a.N);
    return s;
}

// Storage of token j of sequence b: its page, or -1.
__device__ __forceinline__ int kv_page(const KvArgs& a, int b, long long j) {
    if (j < 0 || j >= ((long long)a.max_pages << a.page_shift)) return -1;
    const int page = a.table[b * a.table_stride + (j >> a.page_shift)];
    return (unsigned)page < (unsigned)a.n_pages ? page : -1;
}

// Element offset of row `row0 + i` (new token i of sequence b) in a tensor of new tokens.
__device__ __forceinline__ long long kv_row(const KvArgs& a, const long long* st, int b, long long row0, int i, int h) {
    return (a.cu ? (row0 + i) * st[2] : b * st[0] + i * st[2]) + h * st[1];
}

// Launchers; hipError_t, or -1 for a shape that no kernel was built for.
int launch_kv_append(const KvArgs& a, int dtype, int format, int d, const void* q, const void* k, const void* v,
                     const float* inv_freq, const int* positions, void* q_out, void* k_out, hipStream_t st);
int launch_kv_read(const KvArgs& a, int dtype, int format, int d, void* k_out, void* v_out, hipStream_t st);

// How kv_attn deals the keys out (see AttnArgs), and the workspace that takes.  total: rows of the token axis; longest: of the sequences, as far
// as the caller knows; room: what a sequence can have at most.  fits: the kernels can count the call's work in 32 bits.
struct KvSplit { int groups, splits, whole; size_t ws_bytes; bool fits; };
KvSplit kv_split(int B, int Hq, int Hkv, int N, long long total, int d, int dtype, int format, long long longest, long long room);
int launch_kv_attn(const KvArgs& a, int dtype, int format, int d, const KvSplit& sp, const void* q, void* out, float* lse, float* ws,
                   hipStream_t st);

}  // namespace aa
