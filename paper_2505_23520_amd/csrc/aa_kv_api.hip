// Host side of kv_append, kv_attn and kv_read (include/anchor_attention.h): argument checks and launches.
#include <cmath>
#include <cstring>

#include "../../include/anchor_attention.h"
#include "aa_kv.h"

namespace aa {
namespace {

bool unaligned(const void* ptr) { return ((uintptr_t)ptr & 15) != 0; }

// Strides of a tensor of new tokens: multiples of 16 bytes; `out`: no two rows of it in one place.
int check_rows(const aa_kv_params* p, const int64_t* st, int heads, bool out) {
    const int vec = p->dtype == AA_BF16 ? 8 : 4;
    const int64_t tokens = p->cu_seqlens ? p->total_tokens : p->N;
    for (int e = 0; e < 3; ++e)
        if (!(e == 0 && p->cu_seqlens) && (st[e] < 0 || st[e] % vec || st[e] >= (1ll << 40))) return AA_EINVAL;
    if (!out) return AA_OK;
    if ((tokens > 1 && st[2] < p->d) || (heads > 1 && st[1] < p->d)) return AA_EINVAL;
    if (!p->cu_seqlens && p->B > 1 && st[0] < p->d) return AA_EINVAL;
    return AA_OK;
}

int check_pool(const aa_kv_params* p, const void* pool, const int64_t* st, const uint8_t* sc, const int64_t* ss) {
    const bool fp4 = p->format == AA_KV_FP4;
    const int64_t row = fp4 ? p->d / 2 : p->d, unit = fp4 ? 16 : p->dtype == AA_BF16 ? 8 : 4;
    if (!pool || unaligned(pool)) return AA_EINVAL;
    if (fp4 && (!sc || unaligned(sc))) return AA_EINVAL;
    if (st[0] > (1ll << 60) / p->n_pages || (fp4 && ss[0] > (1ll << 60) / p->n_pages)) return AA_EINVAL;
    // 32-bit byte offsets: the rows of a page, from its first on, and the groups of a row's scales
    const int64_t bytes = fp4 ? 1 : p->dtype == AA_BF16 ? 2 : 4;
    if (st[2] >= (1 << 25) || st[2] * bytes * p->page_size >= (1ll << 31) || (fp4 && ss[2] >= (1 << 28))) return AA_EUNSUPPORTED;
    for (int e = 0; e < 3; ++e) {
        if (st[e] < row || st[e] % unit || st[e] >= (1ll << 40)) return AA_EINVAL;
        if (fp4 && (ss[e] < p->page_size || ss[e] % 16 || ss[e] >= (1ll << 40))) return AA_EINVAL;
    }
    return AA_OK;
}

// What every call has to meet; fills the kernels' arguments.
int make_args(const aa_kv_params* p, KvArgs* a) {
    if (!p) return AA_EINVAL;
    if (p->B <= 0 || p->Hq <= 0 || p->Hkv <= 0 || p->N <= 0 || p->d <= 0) return AA_EINVAL;
    if (p->Hq % p->Hkv != 0) return AA_EINVAL;
    if (p->dtype != AA_FP32 && p->dtype != AA_BF16) return AA_EINVAL;
    if (p->format != AA_KV_PLAIN && p->format != AA_KV_FP4) return AA_EINVAL;
    if (p->page_size <= 0 || (p->page_size & (p->page_size - 1)) || p->n_pages <= 0 || p->max_pages <= 0 || p->max_len < 0) return AA_EINVAL;
    if ((p->causal != 0 && p->causal != 1) || (p->rot_interleaved != 0 && p->rot_interleaved != 1)) return AA_EINVAL;
    if (p->rot_dim < 0 || p->rot_dim > p->d || p->rot_dim % 2) return AA_EINVAL;
    if (std::isnan(p->softmax_scale) || p->softmax_scale < 0.f) return AA_EINVAL;
    if (p->table_stride < p->max_pages || !p->page_table || !p->kv_len) return AA_EINVAL;
    if (p->cu_seqlens && (p->total_tokens <= 0 || p->N > p->total_tokens)) return AA_EINVAL;
    if (p->dtype == AA_BF16 ? p->d != 64 && p->d != 128 : p->d != 32 && p->d != 64 && p->d != 128) return AA_EUNSUPPORTED;
    if (p->format == AA_KV_FP4 && p->dtype != AA_BF16) return AA_EUNSUPPORTED;
    if (p->page_size < 16 || p->page_size > (1 << 20)) return AA_EUNSUPPORTED;
    if (p->rot_dim % 16) return AA_EUNSUPPORTED;
    if ((int64_t)p->max_pages * p->page_size > (1 << 30)) return AA_EUNSUPPORTED;       // tokens of a sequence are counted in 32 bits
    // sequences stand on y of a launch grid, a work-group of 256 threads for every token on x, whose threads are counted in 32 bits
    if (p->B > 65535 || p->Hq > 65535) return AA_EUNSUPPORTED;
    const int64_t tokens = p->cu_seqlens ? p->total_tokens : (int64_t)p->B * p->N;
    if (tokens >= (1 << 24)) return AA_EUNSUPPORTED;
    int rc = check_pool(p, p->kc, p->kc_stride, p->ks, p->ks_stride);
    if (rc == AA_OK) rc = check_pool(p, p->vc, p->vc_stride, p->vs, p->vs_stride);
    if (rc != AA_OK) return rc;

    memset(a, 0, sizeof(*a));
    a->B = p->B; a->Hq = p->Hq; a->Hkv = p->Hkv; a->N = p->N; a->grp = p->Hq / p->Hkv;
    while ((1 << a->page_shift) < p->page_size) ++a->page_shift;
    a->n_pages = p->n_pages; a->max_pages = p->max_pages;
    a->causal = p->causal; a->rot = p->rot_dim; a->interleaved = p->rot_interleaved;
    a->sigma = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)p->d);
    for (int e = 0; e < 3; ++e) {
        a->qs[e] = p->q_stride[e]; a->ks[e] = p->k_stride[e]; a->vs[e] = p->v_stride[e];
        a->os[e] = p->o_stride[e]; a->kos[e] = p->ko_stride[e];
        a->kcs[e] = p->kc_stride[e]; a->vcs[e] = p->vc_stride[e];
        a->kss[e] = p->ks_stride[e]; a->vss[e] = p->vs_stride[e];
    }
    a->kc = (char*)p->kc; a->vc = (char*)p->vc; a->ksc = p->ks; a->vsc = p->vs;
    a->table = p->page_table; a->table_stride = p->table_stride; a->kv_len = p->kv_len;
    a->cu = p->cu_seqlens;
    a->total = tokens;
    return AA_OK;
}

KvSplit split_of(const aa_kv_params* p, const KvArgs& a) {
    const long long room = (long long)p->max_pages * p->page_size;
    return kv_split(p->B, p->Hq, p->Hkv, p->N, a.total, p->d, p->dtype, p->format, p->max_len && p->max_len < room ? p->max_len : room, room);
}

int status_of(int rc, const char* name) {
    if (rc < 0) return AA_EUNSUPPORTED;
    return rc == (int)hipSuccess ? AA_OK : hip_fail((hipError_t)rc, name);
}

}  // namespace
}  // namespace aa

using namespace aa;

extern "C" {

int kv_append(const aa_kv_params* params, const void* q, const void* k, const void* v, const float* inv_freq,
              const int32_t* positions, void* q_out, void* k_out, void* stream) {
    KvArgs a;
    int rc = make_args(params, &a);
    if (rc != AA_OK) return rc;
    if ((q != nullptr) != (q_out != nullptr) || (k != nullptr) != (v != nullptr) || (k_out && !k) || (!q && !k)) return AA_EINVAL;
    if (a.rot && !inv_freq) return AA_EINVAL;
    if (unaligned(q) || unaligned(k) || unaligned(v) || unaligned(q_out) || unaligned(k_out)) return AA_EINVAL;
    if (q && ((rc = check_rows(params, params->q_stride, a.Hq, false)) || (rc = check_rows(params, params->o_stride, a.Hq, true)))) return rc;
    if (k && ((rc = check_rows(params, params->k_stride, a.Hkv, false)) || (rc = check_rows(params, params->v_stride, a.Hkv, false)))) return rc;
    if (k_out && (rc = check_rows(params, params->ko_stride, a.Hkv, true))) return rc;
    return status_of(launch_kv_append(a, params->dtype, params->format, params->d, q, k, v, inv_freq, positions, q_out, k_out,
                                      (hipStream_t)stream), "kv_append_kernel");
}

int kv_attn_workspace_bytes(const aa_kv_params* params, size_t* bytes_out) {
    KvArgs a;
    const int rc = make_args(params, &a);
    if (rc != AA_OK) return rc;
    if (!bytes_out) return AA_EINVAL;
    const KvSplit sp = split_of(params, a);
    if (!sp.fits) return AA_EUNSUPPORTED;
    *bytes_out = sp.ws_bytes;
    return AA_OK;
}

int kv_attn(const aa_kv_params* params, const void* q, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
    KvArgs a;
    int rc = make_args(params, &a);
    if (rc != AA_OK) return rc;
    if (!q || !out || unaligned(q) || unaligned(out) || unaligned(ws)) return AA_EINVAL;
    if ((rc = check_rows(params, params->q_stride, a.Hq, false)) || (rc = check_rows(params, params->o_stride, a.Hq, true))) return rc;
    const KvSplit sp = split_of(params, a);
    if (!sp.fits) return AA_EUNSUPPORTED;
    if (sp.ws_bytes && !ws) return AA_EINVAL;
    if (ws_bytes < sp.ws_bytes) return AA_EWORKSPACE;
    return status_of(launch_kv_attn(a, params->dtype, params->format, params->d, sp, q, out, lse, (float*)ws, (hipStream_t)stream),
                     "kv_attn_kernel");
}

int kv_read(const aa_kv_params* params, void* k_out, void* v_out, void* stream) {
    KvArgs a;
    int rc = make_args(params, &a);
    if (rc != AA_OK) return rc;
    if ((!k_out && !v_out) || unaligned(k_out) || unaligned(v_out)) return AA_EINVAL;
    if (k_out && (rc = check_rows(params, params->k_stride, a.Hkv, true))) return rc;
    if (v_out && (rc = check_rows(params, params->v_stride, a.Hkv, true))) return rc;
    return status_of(launch_kv_read(a, params->dtype, params->format, params->d, k_out, v_out, (hipStream_t)stream), "kv_read_kernel");
}

}  // extern "C"
