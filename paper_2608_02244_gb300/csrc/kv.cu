// kv.cu -- the C ABI of the decode step, prompts and the cache in 4 bits (include/isjl_kv.h): handle, checks, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>

#include "kv_tma.cuh"

struct isjl_kv {
    isjl_kv_config cfg;
    int device = 0;                      // whose memory and kernels these are: calls with another one current are refused
    int sms = 0, shift = 0;
    int per_sm = 0, full = 0;            // the attention's blocks of an SM, with at most `full` queries
    int per_sm4 = 0, full4 = 0;          // attend4's
    // one allocation: the status word, then the workspaces of assign and attend
    unsigned char *d_work = nullptr;
    int32_t *d_status = nullptr;
    int32_t *d_sums = nullptr;
    isjl::CutItem *d_cut = nullptr;
    float2 *d_part_ml = nullptr;
    float *d_part_o = nullptr;
    float2 *d_prefix_ml = nullptr;       // null: this shape has no prefix kernel
    float *d_prefix_o = nullptr;
    void *encoder = nullptr;
};

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMostTokens = INT32_MAX - 255;     // of a request with its prefix: 32-bit places, rounded up to tiles
constexpr int kFiner = 4;     // blocks of the own tokens' kernel for each that fits, beside a prefix's kernel
size_t rounded(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// arrays of numbers lie at multiples of their size
template <typename... T>
bool natural(const T *...p) { return (... && (reinterpret_cast<uintptr_t>(p) % sizeof(T) == 0)); }
// what a copy's map can hold: less than 2^40 bytes
bool stride_ok(int64_t s) { return s > 0 && s % 8 == 0 && s < ((int64_t)1 << 39); }

bool cache_ok(const isjl_kv_cache *c) {
    if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return false;
    for (int i = 0; i < 3; ++i)
        if (!stride_ok(c->k_stride[i]) || !stride_ok(c->v_stride[i])) return false;
    return true;
}

bool cache4_ok(const isjl_kv *kv, const isjl_kv_cache4 *c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) ||
        !aligned16(c->v_scale))
        return false;
    const int64_t numbers = kv->cfg.head_dim / 16 < 8 ? kv->cfg.head_dim / 16 : 8;
    for (int i = 0; i < 3; ++i) {
        for (const int64_t s : {c->k_stride[i], c->v_stride[i]})
            if (s <= 0 || s % 16 != 0 || s >= (int64_t)1 << 40) return false;
        for (const int64_t s : {c->k_scale_stride[i], c->v_scale_stride[i]})
            if (s <= 0 || s % numbers != 0 || s >= (int64_t)1 << 39) return false;
    }
    return true;
}

// Streams and pointers do not say whose they are: stream 0 is that of the current device.
bool device_ok(const isjl_kv *kv) {
    int current = -1;
    if (cudaGetDevice(&current) != cudaSuccess) cudaGetLastError();
    return current == kv->device;
}

// The runtime keeps a failed call's error until it is asked for: the next check of a launch would take it for its own.
isjl_status launched(cudaError_t e) {
    if (e == cudaSuccess) return ISJL_OK;
    cudaGetLastError();
    return ISJL_ERR_CUDA;
}

// what attend and attend4 ask of their arguments, but for the cache
bool attend_ok(const isjl_kv *kv, const isjl_kv_attend_args *a) {
    const int most = !kv ? 0 : kv->cfg.max_rows < ISJL_KV_MAX_ROWS ? kv->cfg.max_rows : ISJL_KV_MAX_ROWS;
    if (!kv || !device_ok(kv) || !a || a->n < 0 || a->n > most || a->table_width < 1 || a->n_table_rows < 0 ||
        a->n_prefix_blocks < 0 || (((int64_t)a->table_width + a->n_prefix_blocks) << kv->shift) > kMostTokens ||
        // slices of 32 tokens are counted in 32 bits
        a->n * ((((int64_t)a->table_width + a->n_prefix_blocks) << kv->shift) / 32 + 2) > INT32_MAX ||
        (a->n_prefix_blocks > 0 && !a->prefix) || a->window < 0 || a->sinks < 0 || !(a->scale > 0.f) || !std::isfinite(a->scale))
        return false;
    if (a->n == 0) return true;
    if (!a->q || !a->out || !a->lens || !a->table || !aligned16(a->q) || !aligned16(a->out) ||
        (!a->rows && a->n > a->n_table_rows) || !natural(a->lse, a->lens, a->rows, a->table, a->prefix))
        return false;
    for (int i = 0; i < 2; ++i)
        if (!stride_ok(a->q_stride[i]) || !stride_ok(a->out_stride[i])) return false;
    return true;
}

// a window as long as any request can be hides nothing
template <typename Args>
void plain_window(const isjl_kv *kv, Args *a) {
    if ((int64_t)a->window >= ((int64_t)a->table_width + a->n_prefix_blocks) << kv->shift) a->window = 0;
    if (a->window == 0) a->sinks = 0;
}

// append and append4: one of the caches is null
isjl_status append_to(isjl_kv *kv, const isjl_kv_append_args *a, const isjl_kv_cache *cache, const isjl_kv_cache4 *cache4,
                      void *stream) {
    if (!kv || !device_ok(kv) || !a || !(cache4 ? cache4_ok(kv, cache4) : cache_ok(cache)) || a->n_tokens < 0 || a->rot < 0 || a->rot > kv->cfg.head_dim || a->rot % 16 != 0 ||
        (a->interleaved != 0 && a->interleaved != 1) || !(a->eps >= 0.f) || !std::isfinite(a->eps))
        return ISJL_ERR_INVALID_ARG;
    if (a->n_tokens == 0) return ISJL_OK;
    const int64_t q_row = (int64_t)kv->cfg.n_q_heads * kv->cfg.head_dim;
    const int64_t row = q_row + 2 * (int64_t)kv->cfg.n_kv_heads * kv->cfg.head_dim;
    if (!a->qkv || !a->q_out || !a->slots || !aligned16(a->qkv) || !aligned16(a->q_out) || !aligned16(a->q_weight) ||
        !aligned16(a->k_weight) || a->qkv_stride < row || a->qkv_stride % 8 != 0 || a->q_out_stride < q_row ||
        a->q_out_stride % 8 != 0 || (a->rot > 0 && (!a->rope || !a->positions || a->n_positions < 1 || !aligned16(a->rope))) ||
        (a->q_out == a->qkv && a->q_out_stride != a->qkv_stride) || !natural(a->positions, a->slots))
        return ISJL_ERR_INVALID_ARG;
    isjl::AppendArgs g;
    std::memset(&g, 0, sizeof(g));
    g.a = *a;
    if (cache4) g.cache4 = *cache4;
    else g.cache = *cache;
    g.n_q_heads = kv->cfg.n_q_heads;
    g.n_kv_heads = kv->cfg.n_kv_heads;
    g.shift = kv->shift;
    g.n_slots = (int64_t)kv->cfg.n_blocks << kv->shift;
    g.status = kv->d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return launched((cache4 ? isjl::launch_append4 : isjl::launch_append)(g, kv->cfg.head_dim, kv->cfg.type, kv->sms, st));
}

// Whether a prefix is done apart, by its own kernel, or read by each query's warps with its own tokens.  The former
// saves n - 1 of n readings of the prefix and costs a launch and the joining of its pieces.  Measured, read against
// apart (32 + 8 heads of 128 values, 256 own tokens): 8 queries over 512 tokens 13.4 and 12.1 us, 16 over 512 15.4 and
// 15.2, 64 over 128 23 and 28, 8 over 2,048 17.2 and 15.0, 64 over 2,048 62 and 30; 4 over 8,192 24.2 and 24.7, 2 over
// 32,768 39 and 38, 4 over 32,768 62 and 39; 64 over 32,768 689 and 73.  The rule goes by queries and tokens alone: of
// these it loses 1.3 and 0.2 us with 8 and 16 over 512, and other head shapes, which save other bytes, were not measured.
bool worth_apart(int n, int tokens) {
    return (int64_t)(n - 1) * tokens >= (n >= 8 ? 12288 : 32768);
}

// Own tokens are bound by memory, the prefix by the tensor cores, and a block of either fills its SM.
//
// A short prefix gets about 64 SMs and own tokens the other 88, which reach nearly the card's bandwidth: both run from
// the start.  Of 0 to 136 SMs for own tokens this was within 7% of the best for eight shapes (4 to 512 requests of 64
// to 8,192 tokens, prefixes of 512 to 8,192), 4 to 28% before one after the other (17 requests over 2,048 tokens 19.2
// and 26.3 us, 128 over 8,192 105 and 140).  The blocks and the prefix's items divide one another where they can,
// since a change of items costs a block about 3 us (64 blocks 43 us where 88 took 52).
//
// Beside a long prefix own tokens get a few SMs, in small runs, and all of them once it is done: 512 requests over
// 32,768 tokens 465 us with 40 SMs, 551 one after the other.  Steps of the prefix's line (256 rows by 128 tokens)
// take 1.4 us with 128 values (taken for 64 too), own tokens run at 60 GB/s an SM.  How long requests are only the device
// knows: they are taken as a quarter of the table's width.  With 512 requests of 256 tokens in the middle and 2,048 at most
// over 32,768 that is right for a table of 2,048 tokens (490 us from a cold L2), and too much for one of 8,192 (822): the
// prefix is taken for the shorter part.
isjl::PrefixLine share_sms(const isjl_kv *kv, const isjl_kv_attend_args *a, int group, int n_kv_heads, int tokens, int *grid) {
    const int sms = kv->sms, per_sm = *grid / sms;
    const isjl::PrefixLine ln = isjl::prefix_line(a->n, group, n_kv_heads, tokens, sms);
    const double own = 0.25 * a->n * ((double)a->table_width * kv->cfg.block_size) * 4.0 * kv->cfg.head_dim * n_kv_heads;
    int blocks = sms * 64 / 152;
    const int even = sms * 72 / 152 / ln.items * ln.items;
    if (even > 0) blocks = even;
    const double prefix = 6e-6 + 1.4e-6 * (double)((ln.work() + blocks - 1) / blocks);
    if (prefix <= 40e-6 || prefix <= own / 5.5e12) {
        const isjl::PrefixLine some = isjl::prefix_line(a->n, group, n_kv_heads, tokens, blocks);
        *grid = per_sm * (sms - some.blocks);
        return some;
    }
    const double all = 6e-6 + 1.4e-6 * (double)((ln.work() + sms - 1) / sms), share = own / (60e9 * all);
    const int most = sms * 40 / 152, left = (share < most ? (int)share : most) / 8 * 8;
    if (left > 0) *grid *= kFiner;
    return isjl::prefix_line(a->n, group, n_kv_heads, tokens, sms - left);
}

}  // namespace

namespace isjl {

void *tensor_map_encoder() {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
        cudaGetLastError();
        return nullptr;
    }
    return fn;
}

namespace {
using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode(void *encoder, CUtensorMap *map, const void *p, int type, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box) {
    const cuuint32_t steps[5] = {1, 1, 1, 1, 1};
    return reinterpret_cast<Encode>(encoder)(
               map, type == ISJL_KV_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void *>(p), dims, strides,
               box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
}  // namespace

bool encode_cache(void *encoder, CUtensorMap *map, void *p, const int64_t *stride, int rows, int halves, int n_blocks, int shift,
                  int n_kv_heads, int head_dim, int type) {
    const cuuint64_t dims[5] = {64, (cuuint64_t)1 << shift, (cuuint64_t)head_dim / 64, (cuuint64_t)n_kv_heads, (cuuint64_t)n_blocks};
    const cuuint64_t strides[4] = {2 * (cuuint64_t)stride[1], 128, 2 * (cuuint64_t)stride[2], 2 * (cuuint64_t)stride[0]};
    const cuuint32_t box[5] = {64, (cuuint32_t)rows, (cuuint32_t)halves, 1, 1};
    return encode(encoder, map, p, type, 5, dims, strides, box);
}

bool encode_queries(void *encoder, CUtensorMap *map, const void *p, const int64_t *stride, int tokens, int heads, int n_tokens, int n_heads,
                    int head_dim, int type) {
    const cuuint64_t dims[4] = {64, (cuuint64_t)head_dim / 64, (cuuint64_t)n_heads, (cuuint64_t)n_tokens};
    const cuuint64_t strides[3] = {128, 2 * (cuuint64_t)stride[1], 2 * (cuuint64_t)stride[0]};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)heads, (cuuint32_t)tokens};
    return encode(encoder, map, p, type, 4, dims, strides, box);
}

}  // namespace isjl

extern "C" {

isjl_status isjl_kv_create(const isjl_kv_config *cfg, isjl_kv **out) {
    if (!out) return ISJL_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || cfg->n_blocks < 1 || cfg->block_size < 8 || cfg->block_size > 256 ||
        (cfg->block_size & (cfg->block_size - 1)) != 0 || cfg->n_kv_heads < 1 || cfg->n_q_heads < cfg->n_kv_heads ||
        cfg->n_q_heads > 1024 || cfg->n_q_heads % cfg->n_kv_heads != 0 ||
        (cfg->head_dim != 64 && cfg->head_dim != 128 && cfg->head_dim != 256) ||
        (cfg->type != ISJL_KV_BF16 && cfg->type != ISJL_KV_FP16) || cfg->max_rows < 1 || cfg->max_rows > (1 << 20))
        return ISJL_ERR_INVALID_ARG;
    isjl_kv *kv = new (std::nothrow) isjl_kv();
    if (!kv) return ISJL_ERR_OOM;
    kv->cfg = *cfg;
    while ((1 << kv->shift) < cfg->block_size) ++kv->shift;
    const int queries = cfg->max_rows < ISJL_KV_MAX_ROWS ? cfg->max_rows : ISJL_KV_MAX_ROWS;
    if (cudaGetDevice(&kv->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, kv->device) != cudaSuccess ||
        isjl::prepare_attend(cfg->head_dim, cfg->type, &kv->per_sm, &kv->full) != cudaSuccess || kv->per_sm < 1) {
        cudaGetLastError();
        delete kv;
        return ISJL_ERR_CUDA;
    }
    int warps4 = 0;
    if (isjl::prepare_attend4(cfg->head_dim, cfg->type, cfg->n_q_heads / cfg->n_kv_heads, kv->sms, &kv->per_sm4, &kv->full4, &warps4) !=
            cudaSuccess || kv->per_sm4 < 1) {
        cudaGetLastError();
        delete kv;
        return ISJL_ERR_CUDA;
    }
    const bool shares = cfg->head_dim <= 128 && cfg->n_q_heads / cfg->n_kv_heads <= 128;
    const size_t sums = rounded(sizeof(int32_t) * (8 + 4 * (size_t)cfg->max_rows));
    const size_t warps = (size_t)kv->per_sm * kv->sms * isjl::kAttendWarps * (shares ? kFiner : 1);
    const int group = cfg->n_q_heads / cfg->n_kv_heads;
    const size_t items = (size_t)queries * cfg->n_kv_heads * ((group + 15) / 16);
    const size_t cuts = rounded(sizeof(isjl::CutItem) * std::max({items, warps, (size_t)warps4}));
    // pieces of attend's and attend4's cut items, 32 rows a warp, or of prompt's
    const size_t cut_rows = std::max({32 * warps, (size_t)32 * warps4, (size_t)isjl::kPromptRows * kv->sms});
    const size_t ml = rounded(sizeof(float2) * cut_rows), o = sizeof(float) * cfg->head_dim * cut_rows;
    // pieces of the prefix part: an item of 256 rows lies in at most sms / items + 2 blocks; and the own tokens' part
    const size_t pieces = shares ? (size_t)kv->sms * 256 + 3 * (size_t)queries * cfg->n_q_heads : 0;
    const size_t prefix_ml = rounded(sizeof(float2) * pieces), prefix_o = sizeof(float) * cfg->head_dim * pieces;
    if (!(kv->encoder = isjl::tensor_map_encoder()) ||
        (shares && isjl::prepare_prefix(cfg->head_dim, cfg->type) != cudaSuccess) ||
        isjl::prepare_prompt(cfg->head_dim, cfg->type) != cudaSuccess) {
        cudaGetLastError();
        delete kv;
        return ISJL_ERR_CUDA;
    }
    const size_t total = kAlign + cuts + sums + ml + rounded(o) + prefix_ml + prefix_o;
    if (cudaMalloc(reinterpret_cast<void **>(&kv->d_work), total) != cudaSuccess) {
        cudaGetLastError();
        delete kv;
        return ISJL_ERR_OOM;
    }
    unsigned char *p = kv->d_work;
    kv->d_status = reinterpret_cast<int32_t *>(p);
    p += kAlign;
    kv->d_cut = reinterpret_cast<isjl::CutItem *>(p);
    p += cuts;
    kv->d_sums = reinterpret_cast<int32_t *>(p);
    p += sums;
    kv->d_part_ml = reinterpret_cast<float2 *>(p);
    p += ml;
    kv->d_part_o = reinterpret_cast<float *>(p);
    p += rounded(o);
    if (shares) {
        kv->d_prefix_ml = reinterpret_cast<float2 *>(p);
        kv->d_prefix_o = reinterpret_cast<float *>(p + prefix_ml);
    }
    // calls may come on any stream: the status word has to be there before create returns
    if (cudaMemset(kv->d_work, 0, kAlign) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
        cudaGetLastError();
        cudaFree(kv->d_work);
        delete kv;
        return ISJL_ERR_CUDA;
    }
    *out = kv;
    return ISJL_OK;
}

void isjl_kv_destroy(isjl_kv *kv) {
    if (!kv) return;
    int current = kv->device;
    cudaGetDevice(&current);
    if (current != kv->device) cudaSetDevice(kv->device);
    cudaDeviceSynchronize();
    cudaFree(kv->d_work);
    if (current != kv->device) cudaSetDevice(current);
    cudaGetLastError();
    delete kv;
}

isjl_status isjl_kv_assign(isjl_kv *kv, const isjl_kv_assign_args *a, void *stream) {
    if (!kv || !device_ok(kv) || !a || a->n_rows < 0 || a->n_rows > kv->cfg.max_rows || a->table_width < 1 ||
        ((int64_t)a->table_width << kv->shift) > INT32_MAX || a->max_tokens < 1 || a->prefix_len < 0 ||
        (int64_t)a->prefix_len + ((int64_t)a->table_width << kv->shift) > INT32_MAX ||
        !a->free_list || !a->n_free || !a->n_free_out || !a->starts || !a->slots || !a->positions || !a->rows || !a->visible ||
        (a->n_rows > 0 && (!a->lens || !a->new_tokens || !a->table || !a->lens_out || !a->granted)) ||
        !natural(a->lens, a->new_tokens, a->table, a->free_list, a->n_free, a->lens_out, a->n_free_out, a->granted, a->starts,
                 a->slots, a->positions, a->rows, a->visible))
        return ISJL_ERR_INVALID_ARG;
    isjl::AssignArgs g;
    std::memset(&g, 0, sizeof(g));
    g.a = *a;
    g.n_blocks = kv->cfg.n_blocks;
    g.shift = kv->shift;
    g.work = kv->d_sums;
    g.status = kv->d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return launched(isjl::launch_assign(g, kv->sms, st));
}

isjl_status isjl_kv_append(isjl_kv *kv, const isjl_kv_append_args *a, const isjl_kv_cache *cache, void *stream) {
    return append_to(kv, a, cache, nullptr, stream);
}

isjl_status isjl_kv_append4(isjl_kv *kv, const isjl_kv_append_args *a, const isjl_kv_cache4 *cache, void *stream) {
    if (!cache) return ISJL_ERR_INVALID_ARG;
    return append_to(kv, a, nullptr, cache, stream);
}

isjl_status isjl_kv_read4(isjl_kv *kv, const isjl_kv_read4_args *a, const isjl_kv_cache4 *cache, void *stream) {
    if (!kv || !device_ok(kv) || !a || !cache4_ok(kv, cache) || a->n_tokens < 0) return ISJL_ERR_INVALID_ARG;
    if (a->n_tokens == 0) return ISJL_OK;
    if (!a->slots || !a->k_out || !a->v_out || !aligned16(a->k_out) || !aligned16(a->v_out) || !natural(a->slots))
        return ISJL_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
        if (!stride_ok(a->k_stride[i]) || !stride_ok(a->v_stride[i])) return ISJL_ERR_INVALID_ARG;
    isjl::Read4Args g;
    std::memset(&g, 0, sizeof(g));
    g.a = *a;
    g.cache = *cache;
    g.n_kv_heads = kv->cfg.n_kv_heads;
    g.shift = kv->shift;
    g.n_slots = (int64_t)kv->cfg.n_blocks << kv->shift;
    g.status = kv->d_status;
    return launched(isjl::launch_read4(g, kv->cfg.head_dim, kv->cfg.type, kv->sms, static_cast<cudaStream_t>(stream)));
}

isjl_status isjl_kv_attend4(isjl_kv *kv, const isjl_kv_attend_args *a, const isjl_kv_cache4 *cache, void *stream) {
    if (!attend_ok(kv, a) || !cache4_ok(kv, cache)) return ISJL_ERR_INVALID_ARG;
    // each query has a place of the line beside its slices
    if (a->n * ((((int64_t)a->table_width + a->n_prefix_blocks) << kv->shift) / 32 + 3) > INT32_MAX) return ISJL_ERR_INVALID_ARG;
    if (a->n == 0) return ISJL_OK;
    isjl::Attend4Args g;
    std::memset(&g, 0, sizeof(g));
    g.a = *a;
    plain_window(kv, &g.a);
    g.cache = *cache;
    g.n_blocks = kv->cfg.n_blocks;
    g.shift = kv->shift;
    g.n_kv_heads = kv->cfg.n_kv_heads;
    g.group = kv->cfg.n_q_heads / kv->cfg.n_kv_heads;
    g.part_o = kv->d_part_o;
    g.part_ml = kv->d_part_ml;
    g.cut = kv->d_cut;
    g.status = kv->d_status;
    const int grid = kv->sms * (a->n <= kv->full4 || kv->per_sm4 == 1 ? kv->per_sm4 : kv->per_sm4 - 1);
    return launched(isjl::launch_attend4(g, kv->cfg.head_dim, kv->cfg.type, grid, static_cast<cudaStream_t>(stream)));
}

isjl_status isjl_kv_prompt(isjl_kv *kv, const isjl_kv_prompt_args *a, const isjl_kv_cache *cache, void *stream) {
    const int most = !kv ? 0 : kv->cfg.max_rows < ISJL_KV_MAX_ROWS ? kv->cfg.max_rows : ISJL_KV_MAX_ROWS;
    if (!kv || !device_ok(kv) || !a || !cache_ok(cache) || a->n_rows < 0 || a->n_rows > most || a->n_tokens < 0 ||
        (int64_t)a->n_tokens * kv->cfg.n_q_heads > INT32_MAX || a->table_width < 1 || a->n_prefix_blocks < 0 ||
        (((int64_t)a->table_width + a->n_prefix_blocks) << kv->shift) > kMostTokens || (a->n_prefix_blocks > 0 && !a->prefix) ||
        a->window < 0 || a->sinks < 0 || !(a->scale > 0.f) || !std::isfinite(a->scale))
        return ISJL_ERR_INVALID_ARG;
    if (a->n_rows == 0 || a->n_tokens == 0) return ISJL_OK;
    if (!a->q || !a->out || !a->starts || !a->lens || !a->table || !aligned16(a->q) || !aligned16(a->out) ||
        !natural(a->lse, a->starts, a->lens, a->table, a->prefix))
        return ISJL_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
        if (!stride_ok(a->q_stride[i]) || !stride_ok(a->out_stride[i])) return ISJL_ERR_INVALID_ARG;
    isjl::PromptArgs g;
    std::memset(&g, 0, sizeof(g));
    g.a = *a;
    plain_window(kv, &g.a);
    g.cache = *cache;
    g.n_blocks = kv->cfg.n_blocks;
    g.shift = kv->shift;
    g.n_kv_heads = kv->cfg.n_kv_heads;
    g.group = kv->cfg.n_q_heads / kv->cfg.n_kv_heads;
    g.part_o = kv->d_part_o;
    g.part_ml = kv->d_part_ml;
    g.cut = reinterpret_cast<isjl::PromptCut *>(kv->d_cut);
    g.status = kv->d_status;
    return launched(isjl::launch_prompt(g, kv->encoder, kv->cfg.head_dim, kv->cfg.type, kv->sms, static_cast<cudaStream_t>(stream)));
}

isjl_status isjl_kv_attend(isjl_kv *kv, const isjl_kv_attend_args *a, const isjl_kv_cache *cache, void *stream) {
    if (!attend_ok(kv, a) || !cache_ok(cache)) return ISJL_ERR_INVALID_ARG;
    if (a->n == 0) return ISJL_OK;
    isjl::AttendArgs g;
    std::memset(&g, 0, sizeof(g));
    g.a = *a;
    plain_window(kv, &g.a);
    g.cache = *cache;
    g.n_blocks = kv->cfg.n_blocks;
    g.shift = kv->shift;
    g.n_kv_heads = kv->cfg.n_kv_heads;
    g.group = kv->cfg.n_q_heads / kv->cfg.n_kv_heads;
    g.part_o = kv->d_part_o;
    g.part_ml = kv->d_part_ml;
    g.cut = kv->d_cut;
    g.status = kv->d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int grid = kv->sms * (a->n <= kv->full || kv->per_sm == 1 ? kv->per_sm : kv->per_sm - 1);
    if (kv->d_prefix_o && g.a.window == 0 && worth_apart(a->n, a->n_prefix_blocks << kv->shift)) {
        isjl::PrefixArgs p;
        std::memset(&p, 0, sizeof(p));
        p.tokens = a->n_prefix_blocks << kv->shift;
        p.line = share_sms(kv, a, g.group, g.n_kv_heads, p.tokens, &grid);
        p.q = a->q;
        p.q_stride[0] = a->q_stride[0];
        p.q_stride[1] = a->q_stride[1];
        p.prefix = a->prefix;
        p.part_o = kv->d_prefix_o;
        p.part_ml = kv->d_prefix_ml;
        p.status = kv->d_status;
        p.scale = a->scale;
        p.n = a->n;
        p.n_blocks = g.n_blocks;
        p.shift = g.shift;
        p.n_kv_heads = g.n_kv_heads;
        p.group = g.group;
        g.line = p.line;
        g.prefix_o = kv->d_prefix_o;
        g.prefix_ml = kv->d_prefix_ml;
        const cudaError_t e = isjl::launch_prefix(p, *cache, kv->encoder, kv->cfg.head_dim, kv->cfg.type, st);
        if (e != cudaSuccess) return launched(e);
    }
    return launched(isjl::launch_attend(g, kv->encoder, kv->cfg.head_dim, kv->cfg.type, grid, st));
}

isjl_status isjl_kv_status(isjl_kv *kv) {
    if (!kv || !device_ok(kv)) return ISJL_ERR_INVALID_ARG;
    // calls may have been replayed from graphs on any stream: all of the device's work is waited for
    int32_t word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&word, kv->d_status, sizeof(word), cudaMemcpyDeviceToHost);
    if (e == cudaSuccess) e = cudaMemset(kv->d_status, 0, sizeof(word));
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return launched(e);
    return word & 2 ? ISJL_ERR_INTERNAL : word ? ISJL_ERR_INVALID_ARG : ISJL_OK;
}

}  // extern "C"
