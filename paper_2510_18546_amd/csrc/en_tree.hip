// Attention over a tree of drafted tokens and the gathered context, and the accepted tokens' way into the contexts.
#include "en_tree_lane.h"

// ---------------------------------------------------------------------------
// tree_attention: one workgroup per (agent, query head, node), 256 keys at a time: a thread takes the score of a key,
// the workgroup their maximum and sum, then a thread one dimension of a part of the keys.
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void tree_attention_kernel(EnTreeArgs a)
{
    __shared__ float sq[D], sp[256], sred[4], sacc[256];
    const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, kvh = hq / (a.Hq / a.Hkv);
    const int done = a.done[b];
    const EnTreeLane mine = tree_lane(a.parent + (size_t)b * a.n, a.n, tree_room(done, a.Nq));
    const unsigned long long way = readlane64(mine.way, i);
    T *out = (T *)a.out + (((size_t)b * a.n + i) * a.Hq + hq) * D;
    if (way == 0) {
        if (tid < D)
            out[tid] = (T)0.f;
        return;
    }
    const int L = a.hdr[4 * b + 1] + done;
    const int pos = L + __builtin_amdgcn_readlane(mine.depth, i);
    if (tid < D / 2) {
        const T *q = (const T *)a.q + (((size_t)b * a.n + i) * a.Hq + hq) * D;
        const float c = a.cos_tab[(size_t)pos * (D / 2) + tid], s = a.sin_tab[(size_t)pos * (D / 2) + tid];
        rope_scale_pair((float)q[tid], (float)q[tid + D / 2], c, s, a.scale_log2e, sq[tid], sq[tid + D / 2]);
    }
    __syncthreads();
    const size_t slab = (size_t)b * a.Hkv + kvh;
    float m = EN_NEG_INF, l = 0.f, acc = 0.f;
    const int d = tid % D, part = tid / D;
    constexpr int PARTS = 256 / D;
    for (int k0 = 0; k0 < L + 64; k0 += 256) {
        // keys 0 .. L - 1: the context; L .. L + 63: the nodes
        const int key = k0 + tid, node = key - L;
        float s = EN_NEG_INF;
        if (node < 0) {
            const T *k = (const T *)a.kc + (slab * a.T + key) * D;
            s = 0.f;
            for (int c = 0; c < D; ++c)
                s += sq[c] * (float)k[c];
        } else if (node < 64 && (way >> node & 1)) {
            const T *k = (const T *)a.k_rows + (((size_t)b * a.n + node) * a.Hkv + kvh) * D;
            const size_t p = L + __popcll(way & ((1ull << node) - 1));
            s = 0.f;
            for (int c = 0; c < D / 2; ++c) {
                float y1, y2;
                rope_key_pair((float)k[c], (float)k[c + D / 2], a.cos_tab[p * (D / 2) + c], a.sin_tab[p * (D / 2) + c], y1, y2);
                s += sq[c] * (float)(T)y1 + sq[c + D / 2] * (float)(T)y2;
            }
        }
        float mx = wave_max(s);
        __syncthreads();
        if (tid % 64 == 0)
            sred[tid / 64] = mx;
        __syncthreads();
        mx = fmaxf(fmaxf(sred[0], sred[1]), fmaxf(sred[2], sred[3]));
        const float now = fmaxf(m, mx), ref = now == EN_NEG_INF ? 0.f : now, keep = fast_exp2(m - ref);
        m = now;
        const float p = s == EN_NEG_INF ? 0.f : fast_exp2(s - ref);
        sp[tid] = p;
        const float ps = wave_sum(p);
        __syncthreads();
        if (tid % 64 == 0)
            sred[tid / 64] = ps;
        __syncthreads();
        l = l * keep + ((sred[0] + sred[1]) + (sred[2] + sred[3]));
        acc *= keep;
        for (int j = part; j < 256; j += PARTS) {
            const int kj = k0 + j, nj = kj - L;
            if (nj < 0) {
                float v;
                if constexpr (sizeof(T) == 4)
                    v = ((const float *)a.vt)[(slab * a.T + kj) * D + d];
                else
                    v = (float)((const T *)a.vt)[(slab * D + d) * a.T + ((kj & ~0xC) | ((kj & 4) << 1) | ((kj & 8) >> 1))];
                acc += sp[j] * v;
            } else if (nj < 64 && (way >> nj & 1)) {
                acc += sp[j] * (float)((const T *)a.v_rows)[(((size_t)b * a.n + nj) * a.Hkv + kvh) * D + d];
            }
        }
    }
    sacc[tid] = acc;
    __syncthreads();
    if (tid < D) {
        float sum = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
            sum += sacc[p * D + tid];
        out[tid] = (T)(sum / l);
    }
}

int en_launch_tree_attention(const en_pool *pool, const EnTreeArgs &a, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const dim3 grid(a.n, a.Hq, a.B), blk(256);
    const int D = pool->d.head_dim;
    if (pool->d.dtype == EN_F32) {
        if (D == 64)
            hipLaunchKernelGGL((tree_attention_kernel<float, 64>), grid, blk, 0, st, a);
        else
            hipLaunchKernelGGL((tree_attention_kernel<float, 128>), grid, blk, 0, st, a);
    } else {
        if (D == 64)
            hipLaunchKernelGGL((tree_attention_kernel<bf16_t, 64>), grid, blk, 0, st, a);
        else
            hipLaunchKernelGGL((tree_attention_kernel<bf16_t, 128>), grid, blk, 0, st, a);
    }
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------
// tree_commit: entry j of an agent's path goes to context row L_c + (done - accepted) + j, the key rotated there. grid:
// (n, Hkv * layers, B), D/2 threads: thread c owns the rotary pair (c, c + D/2).
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(D / 2) void tree_commit_kernel(EnTreeCommitArgs a)
{
    const int j = blockIdx.x, layer = blockIdx.y / a.Hkv, h = blockIdx.y - layer * a.Hkv, b = blockIdx.z;
    const int c = threadIdx.x;
    const int accepted = a.accepted[b], row = a.done[b] - accepted + j;
    const int node = a.path[(size_t)b * a.n + j];
    if (j >= accepted || (unsigned)node >= (unsigned)a.n || (unsigned)row >= (unsigned)a.Nq)
        return;
    const size_t pos = (size_t)a.hdr[4 * b + 1] + row;
    const size_t from = (((size_t)b * a.n + node) * a.Hkv + h) * D, slab = (size_t)b * a.Hkv + h;
    const T *kr = (const T *)a.k_rows[layer] + from, *vr = (const T *)a.v_rows[layer] + from;
    float y1, y2;
    rope_key_pair((float)kr[c], (float)kr[c + D / 2], a.cos_tab[pos * (D / 2) + c], a.sin_tab[pos * (D / 2) + c], y1, y2);
    T *kd = (T *)a.kc[layer] + (slab * a.T + pos) * D;
    kd[c] = (T)y1;
    kd[c + D / 2] = (T)y2;
    if constexpr (sizeof(T) == 4) {
        T *vd = (T *)a.vt[layer] + (slab * a.T + pos) * D;
        vd[c] = vr[c];
        vd[c + D / 2] = vr[c + D / 2];
    } else {
        // transposed layout [D][T], token j in column j with bits 2 and 3 exchanged
        T *vd = (T *)a.vt[layer] + slab * D * a.T + ((pos & ~(size_t)0xC) | ((pos & 4) << 1) | ((pos & 8) >> 1));
        vd[(size_t)c * a.T] = vr[c];
        vd[(size_t)(c + D / 2) * a.T] = vr[c + D / 2];
    }
}

int en_launch_tree_commit(const en_pool *pool, const EnTreeCommitArgs &a, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const int D = pool->d.head_dim;
    const dim3 grid(a.n, a.Hkv * a.layers, a.B), blk(D / 2);
    if (pool->d.dtype == EN_F32) {
        if (D == 64)
            hipLaunchKernelGGL((tree_commit_kernel<float, 64>), grid, blk, 0, st, a);
        else
            hipLaunchKernelGGL((tree_commit_kernel<float, 128>), grid, blk, 0, st, a);
    } else {
        if (D == 64)
            hipLaunchKernelGGL((tree_commit_kernel<bf16_t, 64>), grid, blk, 0, st, a);
        else
            hipLaunchKernelGGL((tree_commit_kernel<bf16_t, 128>), grid, blk, 0, st, a);
    }
    return (int)hipGetLastError();
}
