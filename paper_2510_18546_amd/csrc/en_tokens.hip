// What the next token may be, and which it is: rules on logits, choices, acceptance of a path through a tree.
#include "en_tree_lane.h"

// The rules' arithmetic, every operation rounded to float32 (no fused multiply-add): the choice between near tokens must
// not hang on how an expression was compiled.
__device__ __forceinline__ float ruled(float x, int count, float rep, float freq, float pres)
{
#pragma clang fp contract(off)
    if (count > 0) {
        x = x > 0.f ? x / rep : x * rep;
        x = (x - (float)count * freq) - pres;
    }
    return x;
}

// A logit's rank: larger ones have larger ranks, +0 and -0 the same; 0: NaN or -infinity, which are never chosen.
__device__ __forceinline__ unsigned rank_of(float x)
{
    const unsigned u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u || u == 0xff800000u)
        return 0u;
    return u << 1 == 0u ? 0x80000000u : u >> 31 ? ~u : u | 0x80000000u;
}
// ... with the token, so that the largest word is the largest rank's lowest token.
__device__ __forceinline__ unsigned long long ranked(float x, int token)
{
    const unsigned r = rank_of(x);
    return r ? (unsigned long long)r << 32 | (unsigned)~token : 0ull;
}

// A workgroup takes EN_RULES_CHUNK tokens of a row. grid: (chunks, n, B).
template <typename T, bool CHOOSE>
__global__ __launch_bounds__(256) void rules_kernel(EnRulesArgs a)
{
    __shared__ int count[EN_RULES_CHUNK];
    __shared__ unsigned long long sbest[4];
    const int chunk = blockIdx.x, i = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    unsigned long long way = 0;
    if (a.parent) {
        const EnTreeLane t = tree_lane(a.parent + (size_t)b * a.n, a.n, EN_TREE_MAX_NODES);
        way = readlane64(t.way, i);
        if (way == 0)
            return;
    }
    const int v0 = chunk * EN_RULES_CHUNK, v1 = min(a.vocab, v0 + EN_RULES_CHUNK);
    const en_token_rules &r = a.rules;
    float rep = 1.f, freq = 0.f, pres = 0.f;
    if (r.penalties_dev) {
        rep = r.penalties_dev[3 * b];
        freq = r.penalties_dev[3 * b + 1];
        pres = r.penalties_dev[3 * b + 2];
        for (int k = tid; k < EN_RULES_CHUNK; k += 256)
            count[k] = 0;
        __syncthreads();
        const int h = r.history_dev ? min(max(r.history_len_dev[b], 0), r.history_stride) : 0;
        for (int k = tid; k < h; k += 256) {
            const int v = r.history_dev[(size_t)b * r.history_stride + k];
            if (v >= v0 && v < v1)
                atomicAdd(&count[v - v0], 1);
        }
        if (tid < a.n && tid < 64 && (way >> tid & 1)) {
            const int v = a.tokens[(size_t)b * a.n + tid];
            if (v >= v0 && v < v1)
                atomicAdd(&count[v - v0], 1);
        }
        __syncthreads();
    }
    const size_t row = (size_t)b * a.n + i;
    const T *x = (const T *)a.logits + row * a.logits_stride;
    const float *bias = r.bias_dev ? r.bias_dev + b * r.bias_agent_stride : nullptr;
    const uint32_t *mask = r.mask_dev ? r.mask_dev + b * r.mask_agent_stride + i * r.mask_node_stride : nullptr;
    unsigned long long best = 0;
    for (int v = v0 + tid; v < v1; v += 256) {
        float y = (float)x[v];
        if (r.penalties_dev)
            y = ruled(y, count[v - v0], rep, freq, pres);
        if (bias)
            y += bias[v];
        if (mask && !(mask[v >> 5] >> (v & 31) & 1))
            y = EN_NEG_INF;
        if constexpr (CHOOSE) {
            const unsigned long long w = ranked(y, v);
            best = w > best ? w : best;
        } else {
            ((T *)a.out)[row * a.out_stride + v] = (T)y;
        }
    }
    if constexpr (CHOOSE) {
        for (int s = 32; s > 0; s /= 2) {
            const unsigned long long w = __shfl_xor(best, s, 64);
            best = w > best ? w : best;
        }
        if (tid % 64 == 0)
            sbest[tid / 64] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < 4; ++w)
                best = sbest[w] > best ? sbest[w] : best;
            a.best[row * a.chunks + chunk] = best;
        }
    }
}

// One wave per agent: the choices out of their chunks' best, then the path.
__global__ __launch_bounds__(64) void accept_kernel(EnAcceptArgs a)
{
    const int b = blockIdx.x, lane = threadIdx.x;
    const size_t row = (size_t)b * a.n + lane;
    const int done = a.done[b];
    const EnTreeLane t = tree_lane(a.parent + (size_t)b * a.n, a.n, tree_room(done, a.Nq));
    int choice = -1;
    if (t.present()) {
        if (a.best) {
            unsigned long long best = 0;
            for (int c = 0; c < a.chunks; ++c) {
                const unsigned long long w = a.best[row * a.chunks + c];
                best = w > best ? w : best;
            }
            choice = best ? (int)~(unsigned)best : -1;
        } else {
            choice = a.choice_in[row];
        }
    }
    const int parent = t.present() ? a.parent[row] : -2, token = t.present() ? a.tokens[row] : -1;
    // the path, node by node
    int at = __ballot(lane == 0 && parent == -1) ? 0 : -1, length = 0, next = -1, mine = -1;
    while (at >= 0) {
        if (lane == length)
            mine = at;
        ++length;
        next = __builtin_amdgcn_readlane(choice, at);
        const unsigned long long children = next >= 0 ? __ballot(parent == at && token == next) : 0ull;
        at = children ? __builtin_ctzll(children) : -1;
    }
    if (lane < a.n) {
        a.path[row] = mine;
        if (a.choice_out)
            a.choice_out[row] = choice;
    }
    if (lane == 0) {
        a.accepted[b] = length;
        a.next[b] = next;
        a.done_out[b] = done + length;
    }
}

template <bool CHOOSE>
static int launch_rules(const EnRulesArgs &a, int dtype, void *stream)
{
    const dim3 grid(a.chunks, a.n, a.B), blk(256);
    if (dtype == EN_F32)
        hipLaunchKernelGGL((rules_kernel<float, CHOOSE>), grid, blk, 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL((rules_kernel<bf16_t, CHOOSE>), grid, blk, 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
int en_launch_rules(const EnRulesArgs &a, int dtype, void *stream) { return launch_rules<false>(a, dtype, stream); }
int en_launch_choices(const EnRulesArgs &a, int dtype, void *stream) { return launch_rules<true>(a, dtype, stream); }

int en_launch_accept(const EnAcceptArgs &a, void *stream)
{
    hipLaunchKernelGGL(accept_kernel, dim3(a.B), dim3(64), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
