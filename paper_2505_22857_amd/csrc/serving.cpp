// C ABI entry points of the serving operators that need no language model:
// verification, the paged cache and its pages, and attention.  Argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "trie.h"

namespace ngpu {
size_t verify_workspace(int64_t B, int K, int64_t V);
hipError_t launch_verify(const ngpu_verify_t &a, void *workspace, hipStream_t stream);
hipError_t launch_kv_append(const ngpu_kv_cache_t &c, const ngpu_kv_append_t &a, hipStream_t stream);
size_t attend_workspace(const ngpu_kv_cache_t &c, const ngpu_attend_t &a);
hipError_t launch_attend(const ngpu_kv_cache_t &c, const ngpu_attend_t &a, void *workspace, hipStream_t stream);
size_t attend8_workspace(const ngpu_kv_cache8_t &c, const ngpu_attend_t &a);
hipError_t launch_attend8(const ngpu_kv_cache8_t &c, const ngpu_attend_t &a, void *workspace, hipStream_t stream);
hipError_t launch_kv_append8(const ngpu_kv_cache8_t &c, const ngpu_kv_append_t &a, hipStream_t stream);
hipError_t launch_kv_copy8(const ngpu_kv_cache8_t &c, const int32_t *copies, int64_t n, hipStream_t stream);
size_t kv_fork_workspace(int64_t G, int64_t K, int64_t num_pages);
hipError_t launch_kv_fork(const ngpu_kv_fork_t &a, void *workspace, hipStream_t stream);
hipError_t launch_kv_copy(const ngpu_kv_cache_t &c, const int32_t *copies, int64_t n, hipStream_t stream);
size_t kv_compact_workspace(int64_t num_pages);
hipError_t launch_kv_compact(int32_t *refs, int64_t num_pages, int32_t page_size, int32_t *copies, int32_t *moved,
                             void *workspace, hipStream_t stream);
hipError_t launch_kv_move(int32_t *pages, int64_t rows, int64_t width, int64_t stride, const int32_t *moved,
                          int64_t num_pages, hipStream_t stream);
}  // namespace ngpu

namespace {

int refuse(const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return ngpu::set_error(NGPU_E_INVALID_ARG, buf);
}

int done(hipError_t e, const char *what) {
    if (e == hipSuccess) return ngpu::set_error(NGPU_OK, "");
    return ngpu::set_error(NGPU_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

int check_workspace(const void *p, size_t have, size_t need) {
    if (need == 0) return NGPU_OK;
    if (!p || have < need) return refuse("the workspace has %zu bytes, %zu are needed", p ? have : 0, need);
    if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return refuse("the workspace must be 16-byte aligned");
    return NGPU_OK;
}

// Rows times elements of a call: every index fits 62 bits.
constexpr int64_t kMostElements = int64_t(1) << 40;

int check_verify(const ngpu_verify_t *a) {
    if (!a) return refuse("null argument");
    if (a->B < 0 || a->B > NGPU_LM_MAX_SEQUENCES) return refuse("B = %lld outside [0, %d]", (long long)a->B,
                                                                NGPU_LM_MAX_SEQUENCES);
    if (a->K < 0 || a->K > NGPU_LM_MAX_DRAFT) return refuse("K = %d outside [0, %d]", a->K, NGPU_LM_MAX_DRAFT);
    if (a->V < 1 || a->V > INT32_MAX) return refuse("V = %lld outside [1, 2^31 - 1]", (long long)a->V);
    if (a->dtype != NGPU_F32 && a->dtype != NGPU_F16 && a->dtype != NGPU_BF16)
        return refuse("unknown type %d of the logits", a->dtype);
    const float t = a->temperature;
    if (t != 0.0f && !(std::isfinite(t) && t >= NGPU_LM_MIN_TEMPERATURE))
        return refuse("temperature must be 0 or finite and at least %g", NGPU_LM_MIN_TEMPERATURE);
    return NGPU_OK;
}

int check_cache(const ngpu_kv_cache_t *c) {
    if (!c) return refuse("null argument");
    if (c->dtype != NGPU_F16 && c->dtype != NGPU_BF16) return refuse("the cache holds half or bfloat16 values");
    if (c->dim < 1 || c->dim > NGPU_LM_MAX_HEAD_DIM)
        return refuse("dim = %d outside [1, %d]", c->dim, NGPU_LM_MAX_HEAD_DIM);
    if (c->heads < 1 || c->heads > 65536) return refuse("heads = %d outside [1, 65536]", c->heads);
    if (c->page_size < 1) return refuse("page_size = %d must be positive", c->page_size);
    if (c->num_pages < 0 || c->num_pages > INT32_MAX) return refuse("num_pages = %lld out of range",
                                                                    (long long)c->num_pages);
    if (c->k_stride_page < 0 || c->k_stride_token < 0 || c->k_stride_head < 0 || c->v_stride_page < 0 ||
        c->v_stride_token < 0 || c->v_stride_head < 0)
        return refuse("negative strides of the cache");
    if (c->num_pages > 0 && (!c->k || !c->v)) return refuse("null device pointer of the cache");
    return NGPU_OK;
}

int check_cache8(const ngpu_kv_cache8_t *c) {
    if (!c) return refuse("null argument");
    if (const int rc = check_cache(&c->cache)) return rc;
    if (c->block < 1 || c->block > NGPU_LM_MAX_SCALE_BLOCK || c->cache.page_size % c->block != 0)
        return refuse("block = %d must lie in [1, %d] and divide a page of %d tokens", c->block, NGPU_LM_MAX_SCALE_BLOCK,
                      c->cache.page_size);
    if (c->k_scale_stride_page < 0 || c->k_scale_stride_block < 0 || c->k_scale_stride_head < 0 ||
        c->v_scale_stride_page < 0 || c->v_scale_stride_block < 0 || c->v_scale_stride_head < 0)
        return refuse("negative strides of the scales");
    if (c->cache.num_pages > 0 && (!c->k_scale || !c->v_scale)) return refuse("null device pointer of the scales");
    return NGPU_OK;
}

// Dimensions of a strided tensor: entries, and the elements from one to the next.
struct Axes {
    struct {
        int64_t size, stride;
    } at[4];
    int count = 0;
};

// Whether no two indexes share an element, for tensors whose dimensions are nested in any order, with gaps or not: from the
// smallest stride on, each passes what the dimensions before span.
bool apart(Axes axes) {
    std::sort(axes.at, axes.at + axes.count, [](const auto &a, const auto &b) { return a.stride < b.stride; });
    __int128 span = 0;
    for (int i = 0; i < axes.count; ++i) {
        if (axes.at[i].size <= 1) continue;
        if (axes.at[i].stride <= span) return false;
        span += __int128(axes.at[i].size - 1) * axes.at[i].stride;
    }
    return true;
}

// Scales that a call writes: each needs its own element, among keys', among values' and between the two.  With `same`, writers
// of one element write one value, so a stride of 0, and one tensor for both, do no harm.
int check_scales_apart(const ngpu_kv_cache8_t &c, bool same) {
    if (c.cache.num_pages == 0) return NGPU_OK;
    const int64_t sizes[] = {c.cache.num_pages, c.cache.page_size / c.block, c.cache.heads};
    const int64_t strides[2][3] = {{c.k_scale_stride_page, c.k_scale_stride_block, c.k_scale_stride_head},
                                   {c.v_scale_stride_page, c.v_scale_stride_block, c.v_scale_stride_head}};
    Axes axes[2];
    __int128 bytes[2] = {4, 4};   // from the first scale to behind the last
    bool alike = true;
    for (int i = 0; i < 3; ++i) {
        alike = alike && (sizes[i] <= 1 || strides[0][i] == strides[1][i]);
        for (int t = 0; t < 2; ++t) {
            if (!same || strides[t][i] > 0) axes[t].at[axes[t].count++] = {sizes[i], strides[t][i]};
            bytes[t] += __int128(sizes[i] - 1) * strides[t][i] * 4;
        }
    }
    for (int t = 0; t < 2; ++t)
        if (!apart(axes[t])) return refuse("%s_scale is written and must not overlap itself", t == 0 ? "k" : "v");
    const uintptr_t k = reinterpret_cast<uintptr_t>(c.k_scale), v = reinterpret_cast<uintptr_t>(c.v_scale);
    const uintptr_t between = k < v ? v - k : k - v;
    if (between >= bytes[k < v ? 0 : 1] || (same && alike && between == 0)) return NGPU_OK;
    axes[0].at[axes[0].count++] = {2, int64_t(between / 4)};
    if (!alike || between % 4 != 0 || !apart(axes[0])) return refuse("k_scale and v_scale are written and must not overlap");
    return NGPU_OK;
}

int check_rows(int64_t S, int64_t T, int64_t heads, int64_t dim) {
    if (S < 0 || S > NGPU_LM_MAX_SEQUENCES) return refuse("S = %lld outside [0, %d]", (long long)S,
                                                          NGPU_LM_MAX_SEQUENCES);
    if (T < 0 || T > INT32_MAX) return refuse("T = %lld outside [0, 2^31 - 1]", (long long)T);
    if (heads < 0 || heads > 65536) return refuse("q_heads = %lld out of range", (long long)heads);
    if (S > 0 && T > 0 && S * T > kMostElements / (heads + 1) / dim) return refuse("the call is too large");
    return NGPU_OK;
}

// `a`: the arguments as the kernels take them; `empty`: there is nothing to append.
int check_append(const ngpu_kv_cache_t &c, const ngpu_kv_append_t *args, ngpu_kv_append_t &a, bool &empty) {
    if (!args) return refuse("null argument");
    a = *args;
    if (!a.q) a.q_heads = 0;
    if (const int rc = check_rows(a.S, a.T, int64_t(a.q_heads) + 2 * c.heads, c.dim)) return rc;
    if (a.q && a.q_heads < 1) return refuse("q_heads = %d must be positive", a.q_heads);
    if (a.k_stride_seq < 0 || a.k_stride_token < 0 || a.k_stride_head < 0 || a.v_stride_seq < 0 ||
        a.v_stride_token < 0 || a.v_stride_head < 0 ||
        (a.q && (a.q_stride_seq < 0 || a.q_stride_token < 0 || a.q_stride_head < 0)))
        return refuse("negative strides");
    if (a.pages_width < 0 || a.pages_width > INT32_MAX || a.pages_stride < 0) return refuse("bad page tables");
    if (a.rotary < 0 || a.rotary > c.dim || a.rotary % 2 != 0)
        return refuse("rotary = %d must be even and lie in [0, %d]", a.rotary, c.dim);
    if (a.layout != NGPU_ROPE_HALF && a.layout != NGPU_ROPE_INTERLEAVED)
        return refuse("unknown rotation layout %d", a.layout);
    empty = a.S == 0 || a.T == 0;
    if (empty) return NGPU_OK;
    if (!a.k || !a.v || !a.start || (!a.pages && a.pages_width > 0) || (a.q && !a.q_out) ||
        (a.rotary > 0 && a.positions_count > 0 && (!a.cos || !a.sin)))
        return refuse("null device pointer");
    if (a.q && a.q_out == a.q) return refuse("q_out must not overlap q");
    return NGPU_OK;
}

int check_attend(const ngpu_kv_cache_t *c, const ngpu_attend_t *a) {
    if (const int rc = check_cache(c)) return rc;
    if (!a) return refuse("null argument");
    if (const int rc = check_rows(a->S, a->T, a->q_heads, c->dim)) return rc;
    if (a->q_heads < 1 || a->q_heads % c->heads != 0)
        return refuse("q_heads = %d is no multiple of the cache's %d heads", a->q_heads, c->heads);
    if (a->G < 0 || (a->G > 0 && a->S % a->G != 0))
        return refuse("%lld sequences do not divide into %lld groups", (long long)a->S, (long long)a->G);
    if (a->G > 0 && (a->prefix_width < 0 || a->prefix_width > INT32_MAX || a->prefix_stride < 0))
        return refuse("bad prefix tables");
    if (a->pages && (a->pages_width < 0 || a->pages_width > INT32_MAX || a->pages_stride < 0))
        return refuse("bad page tables");
    if (a->q_stride_seq < 0 || a->q_stride_token < 0 || a->q_stride_head < 0) return refuse("negative strides");
    if (!std::isfinite(a->scale)) return refuse("scale must be finite");
    return NGPU_OK;
}

int check_attend_pointers(const ngpu_attend_t &a) {
    if (!a.q || !a.out || (a.G > 0 && (!a.prefix_lengths || (a.prefix_width > 0 && !a.prefix_pages))) ||
        (a.pages && !a.lengths))
        return refuse("null device pointer");
    return NGPU_OK;
}

int check_pool(int64_t num_pages, int32_t page_size) {
    if (num_pages < 0 || num_pages > NGPU_LM_MAX_PAGES)
        return refuse("num_pages = %lld outside [0, %lld]", (long long)num_pages, (long long)NGPU_LM_MAX_PAGES);
    if (page_size < 1) return refuse("page_size = %d must be positive", page_size);
    return NGPU_OK;
}

bool fork_sizes(int64_t G, int64_t W, int64_t K) {
    return G >= 0 && G <= NGPU_LM_MAX_SEQUENCES && W >= 0 && W <= NGPU_LM_MAX_FORK && K >= 0 && K <= NGPU_LM_MAX_FORK &&
           G * W <= NGPU_LM_MAX_SEQUENCES && G * K <= NGPU_LM_MAX_SEQUENCES;
}

int check_fork(const ngpu_kv_fork_t *a) {
    if (!a) return refuse("null argument");
    if (!fork_sizes(a->G, a->W, a->K))
        return refuse("G = %lld, W = %lld, K = %lld: W and K lie in [0, %d], G W and G K in [0, %d]", (long long)a->G,
                      (long long)a->W, (long long)a->K, NGPU_LM_MAX_FORK, NGPU_LM_MAX_SEQUENCES);
    if (const int rc = check_pool(a->num_pages, a->page_size)) return rc;
    if (a->width < 0 || a->width > INT32_MAX || a->pages_stride < 0) return refuse("bad page tables");
    if (a->T < 0 || a->T > INT32_MAX) return refuse("T = %lld outside [0, 2^31 - 1]", (long long)a->T);
    if (a->G * (a->W + a->K) > 0 && a->width > kMostElements / (a->G * (a->W + a->K))) return refuse("the call is too large");
    return NGPU_OK;
}

}  // namespace

extern "C" {

size_t ngpu_lm_verify_workspace(int64_t B, int32_t K, int64_t V) {
    if (B <= 0 || B > NGPU_LM_MAX_SEQUENCES || K < 0 || K > NGPU_LM_MAX_DRAFT || V < 1 || V > INT32_MAX) return 0;
    return ngpu::verify_workspace(B, K, V);
}

int ngpu_lm_verify(const ngpu_verify_t *args, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_verify(args)) return rc;
    const ngpu_verify_t &a = *args;
    if (a.B == 0) return done(hipSuccess, "");
    const bool sample = a.temperature != 0.0f;
    if (!a.logits || !a.out_tokens || !a.accepted || (a.K > 0 && !a.tokens) || (a.states && !a.draft_states) ||
        (sample && (!a.noise || (a.K > 0 && !a.uniforms))))
        return refuse("null device pointer");
    if (a.logits_stride_b < 0 || a.logits_stride_k < 0 || (sample && a.noise_stride_b < 0) ||
        (sample && a.logprobs && (a.logprobs_stride_b < 0 || a.logprobs_stride_k < 0)))
        return refuse("negative strides");
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu::verify_workspace(a.B, a.K, a.V))) return rc;
    return done(ngpu::launch_verify(a, d_workspace, static_cast<hipStream_t>(hip_stream)), "verify launch");
}

int ngpu_lm_kv_append(const ngpu_kv_cache_t *cache, const ngpu_kv_append_t *args, void *hip_stream) {
    if (const int rc = check_cache(cache)) return rc;
    ngpu_kv_append_t a;
    bool empty;
    if (const int rc = check_append(*cache, args, a, empty)) return rc;
    if (empty) return done(hipSuccess, "");
    return done(ngpu::launch_kv_append(*cache, a, static_cast<hipStream_t>(hip_stream)), "append launch");
}

int ngpu_lm_kv_append8(const ngpu_kv_cache8_t *cache, const ngpu_kv_append_t *args, void *hip_stream) {
    if (const int rc = check_cache8(cache)) return rc;
    ngpu_kv_append_t a;
    bool empty;
    if (const int rc = check_append(cache->cache, args, a, empty)) return rc;
    if (empty) return done(hipSuccess, "");
    if (const int rc = check_scales_apart(*cache, false)) return rc;
    return done(ngpu::launch_kv_append8(*cache, a, static_cast<hipStream_t>(hip_stream)), "append launch");
}

size_t ngpu_lm_attend_workspace(const ngpu_kv_cache_t *cache, const ngpu_attend_t *args) {
    if (check_attend(cache, args) != NGPU_OK) return 0;
    if (args->S == 0 || args->T == 0) return 0;
    return ngpu::attend_workspace(*cache, *args);
}

int ngpu_lm_attend(const ngpu_kv_cache_t *cache, const ngpu_attend_t *args, void *d_workspace,
                   size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_attend(cache, args)) return rc;
    const ngpu_attend_t &a = *args;
    if (a.S == 0 || a.T == 0) return done(hipSuccess, "");
    if (const int rc = check_attend_pointers(a)) return rc;
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu::attend_workspace(*cache, a))) return rc;
    return done(ngpu::launch_attend(*cache, a, d_workspace, static_cast<hipStream_t>(hip_stream)), "attend launch");
}

size_t ngpu_lm_attend8_workspace(const ngpu_kv_cache8_t *cache, const ngpu_attend_t *args) {
    if (check_cache8(cache) != NGPU_OK || check_attend(&cache->cache, args) != NGPU_OK) return 0;
    if (args->S == 0 || args->T == 0) return 0;
    return ngpu::attend8_workspace(*cache, *args);
}

int ngpu_lm_attend8(const ngpu_kv_cache8_t *cache, const ngpu_attend_t *args, void *d_workspace,
                    size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_cache8(cache)) return rc;
    if (const int rc = check_attend(&cache->cache, args)) return rc;
    const ngpu_attend_t &a = *args;
    if (a.S == 0 || a.T == 0) return done(hipSuccess, "");
    if (const int rc = check_attend_pointers(a)) return rc;
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu::attend8_workspace(*cache, a))) return rc;
    return done(ngpu::launch_attend8(*cache, a, d_workspace, static_cast<hipStream_t>(hip_stream)), "attend launch");
}

size_t ngpu_lm_kv_fork_workspace(int64_t G, int64_t K, int64_t num_pages) {
    if (!fork_sizes(G, 0, K) || num_pages < 0 || num_pages > NGPU_LM_MAX_PAGES || G * K == 0) return 0;
    return ngpu::kv_fork_workspace(G, K, num_pages);
}

int ngpu_lm_kv_fork(const ngpu_kv_fork_t *args, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_fork(args)) return rc;
    const ngpu_kv_fork_t &a = *args;
    const bool old = a.G * a.W > 0, made = a.G * a.K > 0;
    if (!old && !made) return done(hipSuccess, "");
    if ((old && (!a.lengths || (a.width > 0 && !a.pages))) || (a.num_pages > 0 && !a.refs) ||
        (made && (!a.parents || !a.out_lengths || !a.copies || (a.width > 0 && !a.out_pages))))
        return refuse("null device pointer");
    if (a.out_pages && a.out_pages == a.pages) return refuse("out_pages must not overlap pages");
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu_lm_kv_fork_workspace(a.G, a.K, a.num_pages)))
        return rc;
    return done(ngpu::launch_kv_fork(a, d_workspace, static_cast<hipStream_t>(hip_stream)), "fork launch");
}

int ngpu_lm_kv_copy(const ngpu_kv_cache_t *cache, const int32_t *copies, int64_t n, void *hip_stream) {
    if (const int rc = check_cache(cache)) return rc;
    if (n < 0 || n > NGPU_LM_MAX_PAGES) return refuse("n = %lld out of range", (long long)n);
    if (n == 0 || cache->num_pages == 0) return done(hipSuccess, "");
    if (!copies) return refuse("null device pointer");
    return done(ngpu::launch_kv_copy(*cache, copies, n, static_cast<hipStream_t>(hip_stream)), "copy launch");
}

int ngpu_lm_kv_copy8(const ngpu_kv_cache8_t *cache, const int32_t *copies, int64_t n, void *hip_stream) {
    if (const int rc = check_cache8(cache)) return rc;
    if (n < 0 || n > NGPU_LM_MAX_PAGES) return refuse("n = %lld out of range", (long long)n);
    if (n == 0 || cache->cache.num_pages == 0) return done(hipSuccess, "");
    if (!copies) return refuse("null device pointer");
    if (const int rc = check_scales_apart(*cache, true)) return rc;
    return done(ngpu::launch_kv_copy8(*cache, copies, n, static_cast<hipStream_t>(hip_stream)), "copy launch");
}

size_t ngpu_lm_kv_compact_workspace(int64_t num_pages) {
    return num_pages <= 0 || num_pages > NGPU_LM_MAX_PAGES ? 0 : ngpu::kv_compact_workspace(num_pages);
}

int ngpu_lm_kv_compact(int32_t *refs, int64_t num_pages, int32_t page_size, int32_t *copies, int32_t *moved,
                       void *d_workspace, size_t workspace_bytes, void *hip_stream) {
    if (const int rc = check_pool(num_pages, page_size)) return rc;
    if (num_pages == 0) return done(hipSuccess, "");
    if (!refs || !moved || (num_pages > 1 && !copies)) return refuse("null device pointer");
    if (const int rc = check_workspace(d_workspace, workspace_bytes, ngpu::kv_compact_workspace(num_pages))) return rc;
    return done(ngpu::launch_kv_compact(refs, num_pages, page_size, copies, moved, d_workspace,
                                        static_cast<hipStream_t>(hip_stream)), "compaction launch");
}

int ngpu_lm_kv_move(int32_t *pages, int64_t rows, int64_t width, int64_t pages_stride, const int32_t *moved,
                    int64_t num_pages, void *hip_stream) {
    if (const int rc = check_pool(num_pages, 1)) return rc;
    if (rows < 0 || width < 0 || width > INT32_MAX || rows > kMostElements / (width + 1)) return refuse("bad page tables");
    if (rows > 1 && pages_stride < width) return refuse("the rows of a page table must not overlap");
    if (rows == 0 || width == 0 || num_pages == 0) return done(hipSuccess, "");
    if (!pages || !moved) return refuse("null device pointer");
    return done(ngpu::launch_kv_move(pages, rows, width, pages_stride, moved, num_pages,
                                     static_cast<hipStream_t>(hip_stream)), "move launch");
}

}  // extern "C"
