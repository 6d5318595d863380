// Attention of a tree of drafted tokens over a paged cache and the tree itself.
#include <limits.h>
#include <math.h>

#include <cuda_fp16.h>

#include "spec_common.cuh"

namespace spec {

namespace {

constexpr int kSimpleThreads = 128;

template <int kDtype> __device__ __forceinline__ float to_float(uint16_t x) {
    return kDtype == SPEC_BF16 ? bf16_bits_to_float(x) : __half2float(__ushort_as_half(x));
}
template <int kDtype> __device__ __forceinline__ uint16_t from_float(float x) {
    return kDtype == SPEC_BF16 ? (uint16_t)float_to_bf16_bits(x) : __half_as_ushort(__float2half_rn(x));
}

template <bool kMax>
__device__ float block_reduce(float x, float *part) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float y = __shfl_xor_sync(0xffffffffu, x, off);
        x = kMax ? fmaxf(x, y) : x + y;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = part[0];
    for (int i = 1; i < kSimpleThreads / 32; ++i) x = kMax ? fmaxf(x, part[i]) : x + part[i];
    return x;
}

// One CTA per (query head, node, sequence): a thread per key for the scores, a thread per column for the sum of the values.
template <int kDtype>
__global__ void __launch_bounds__(kSimpleThreads) tree_attention_kernel(const spec_tree_attention_t a) {
    __shared__ float q[128], p[kSimpleThreads], part[kSimpleThreads / 32];
    __shared__ const uint16_t *val[kSimpleThreads];
    griddep_launch();
    griddep_wait();
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, t = threadIdx.x, g = h / (a.Hq / a.Hkv);
    const int cap = (int)min((long long)a.max_pages * a.page_size, (long long)INT_MAX);
    const int len_in = a.seq_len[b], nodes_in = a.n_nodes ? a.n_nodes[b] : a.T;
    const int len = min(max(len_in, 0), cap), nodes = min(max(nodes_in, 0), a.T);
    if (t == 0 && (len != len_in || nodes != nodes_in)) report_error(a.err_word, SPEC_ERR_INDEX_RANGE);
    if (i >= nodes) return;
    const uint16_t *qr = (const uint16_t *)a.q + b * a.q_stride[0] + i * a.q_stride[1] + h * a.q_stride[2];
    if (t < a.D) q[t] = to_float<kDtype>(qr[t]);
    float top = -INFINITY, total = 0.f, acc = 0.f;
    for (int k0 = 0; k0 < len + nodes; k0 += kSimpleThreads) {
        __syncthreads();
        const int key = k0 + t;
        const uint16_t *kr = nullptr, *vr = nullptr;
        if (key < len) {
            const int page = key / a.page_size, off = key - page * a.page_size, id = a.block_table[b * a.table_stride + page];
            if (id >= 0 && id < a.n_pages) {
                kr = (const uint16_t *)a.k_cache + id * a.kc_stride[0] + off * a.kc_stride[1] + g * a.kc_stride[2];
                vr = (const uint16_t *)a.v_cache + id * a.vc_stride[0] + off * a.vc_stride[1] + g * a.vc_stride[2];
            } else {
                report_error(a.err_word, SPEC_ERR_INDEX_RANGE);
            }
        } else if (key < len + nodes) {
            const int n = key - len;
            kr = (const uint16_t *)a.k + b * a.k_stride[0] + n * a.k_stride[1] + g * a.k_stride[2];
            vr = (const uint16_t *)a.v + b * a.v_stride[0] + n * a.v_stride[1] + g * a.v_stride[2];
        }
        bool sees = key < len;
        if (key >= len && key < len + nodes) {
            const int n = key - len;
            sees = a.mask ? a.mask[((size_t)b * a.T + i) * ((a.T + 31) / 32) + (n >> 5)] >> (n & 31) & 1 : n <= i;
        }
        float s = -INFINITY;
        if (sees) {
            s = 0.f;
            if (kr)
                for (int d = 0; d < a.D; ++d) s += q[d] * to_float<kDtype>(kr[d]);
            s *= a.scale;
        }
        const float m = fmaxf(top, block_reduce<true>(s, part));
        const float w = sees ? expf(s - m) : 0.f;
        p[t] = w;
        val[t] = sees ? vr : nullptr;
        const float keep = m == -INFINITY ? 1.f : expf(top - m);
        total = total * keep + block_reduce<false>(w, part);
        acc *= keep;
        top = m;
        if (t < a.D)
            for (int j = 0; j < min(kSimpleThreads, len + nodes - k0); ++j)
                if (val[j]) acc += p[j] * to_float<kDtype>(val[j][t]);
    }
    uint16_t *out = (uint16_t *)a.out + b * a.out_stride[0] + i * a.out_stride[1] + h * a.out_stride[2];
    if (t < a.D) out[t] = from_float<kDtype>(total == 0.f ? 0.f : acc / total);
    if (t == 0 && a.lse) a.lse[((size_t)b * a.T + i) * a.Hq + h] = total == 0.f ? -INFINITY : top + logf(total);
}

}  // namespace
}  // namespace spec

using namespace spec;

namespace {

bool strides_ok(const int64_t (&s)[3]) { return s[0] >= 0 && s[1] >= 0 && s[2] >= 0 && !(s[0] % 8) && !(s[1] % 8) && !(s[2] % 8); }

int check_shape(int B, int T, int Hq, int Hkv, int D) {
    if (B <= 0 || T <= 0 || Hq <= 0 || Hkv <= 0 || D <= 0) return SPEC_ERR_INVALID_ARG;
    if (D % 8 != 0 || D > 128 || Hq % Hkv != 0 || T > SPEC_MAX_TREE_NODES || B > 65535 || Hq > 65535) return SPEC_ERR_SHAPE;
    return SPEC_OK;
}

}  // namespace

extern "C" {

size_t spec_tree_attention_workspace_bytes(int B, int T, int Hq, int Hkv, int D) {
    if (check_shape(B, T, Hq, Hkv, D) != SPEC_OK) return 0;
    return kWsAlign;
}

int spec_tree_attention(const spec_tree_attention_t *a, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!a || !a->q || !a->k || !a->v || !a->k_cache || !a->v_cache || !a->block_table || !a->seq_len || !a->out)
        return SPEC_ERR_INVALID_ARG;
    if (a->dtype != SPEC_BF16 && a->dtype != SPEC_F16) return SPEC_ERR_INVALID_ARG;
    const int rc = check_shape(a->B, a->T, a->Hq, a->Hkv, a->D);
    if (rc != SPEC_OK) return rc;
    if (a->page_size <= 0 || a->n_pages <= 0 || a->max_pages <= 0 || !(a->scale == a->scale)) return SPEC_ERR_INVALID_ARG;
    if (a->table_stride < a->max_pages) return SPEC_ERR_SHAPE;
    const void *ptrs[] = {a->q, a->k, a->v, a->k_cache, a->v_cache, a->out};
    for (const void *p : ptrs)
        if ((uintptr_t)p % 16 != 0) return SPEC_ERR_INVALID_ARG;
    if (!strides_ok(a->q_stride) || !strides_ok(a->k_stride) || !strides_ok(a->v_stride) || !strides_ok(a->kc_stride) ||
        !strides_ok(a->vc_stride) || !strides_ok(a->out_stride))
        return SPEC_ERR_SHAPE;
    if (!workspace || ((uintptr_t)workspace % kWsAlign) != 0 ||
        workspace_bytes < spec_tree_attention_workspace_bytes(a->B, a->T, a->Hq, a->Hkv, a->D))
        return SPEC_ERR_WORKSPACE;
    const dim3 grid(a->Hq, a->T, a->B);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a->dtype == SPEC_BF16) SPEC_CUDA_TRY(launch_pdl(tree_attention_kernel<SPEC_BF16>, grid, dim3(kSimpleThreads), 0, st, *a));
    else SPEC_CUDA_TRY(launch_pdl(tree_attention_kernel<SPEC_F16>, grid, dim3(kSimpleThreads), 0, st, *a));
    return SPEC_OK;
}

}  // extern "C"
