// What the next token may be, and which it is: rules on logits, choices, acceptance of a path through a tree.
#include "en_tree_lane.h"

// The rules' arithmetic, every operation rounded to float32 (no fused multiply-add): the choice between near tokens must
// not hang on how an expression was compiled.
__device__ __forceinline__ float penalised(float x, int count, float rep, float freq, float pres)
{
#pragma clang fp contract(off)
    x = x > 0.f ? x / rep : x * rep;
    return (x - (float)count * freq) - pres;
}

// A logit's rank: larger ones have larger ranks, +0 and -0 the same. (Never of NaN or -infinity, whose rank is 0: they
// are not chosen.)
__device__ __forceinline__ unsigned rank_of(float x)
{
    const unsigned u = __float_as_uint(x);
    return u << 1 == 0u ? 0x80000000u : u >> 31 ? ~u : u | 0x80000000u;
}

template <typename F>
__device__ __forceinline__ unsigned wave_reduce(unsigned v, F op)
{
    return __float_as_uint(lanes_reduce<64>(__uint_as_float(v), [op](float x, float y) {
        return __uint_as_float(op(__float_as_uint(x), __float_as_uint(y)));
    }));
}
// The largest rank of the wave's lanes and the lowest token that has it, as one word whose order is the choice's; 0: none.
__device__ __forceinline__ unsigned long long wave_choice(unsigned rank, int token)
{
    const unsigned top = wave_reduce(rank, [](unsigned x, unsigned y) { return x > y ? x : y; });
    const unsigned first = wave_reduce(rank == top ? (unsigned)token : ~0u, [](unsigned x, unsigned y) { return x < y ? x : y; });
    return top ? (unsigned long long)top << 32 | ~first : 0ull;
}

// Order of a wave's own LDS accesses by different lanes, which the hardware keeps.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------------------
// rules: a workgroup takes EN_RULES_CHUNK tokens of `a.nodes` of an agent's rows, a wave a quarter of the tokens of each
// row: 16 a lane, in two runs of eight. Bound by reading the logits once (and writing them once).
//
// The tokens that penalties concern are few: they are counted into a table in LDS once for all rows of the workgroup, each
// wave lists those of its quarter, and in a row only they are divided and subtracted from, in a copy of the quarter in
// LDS (a division for every token would be 12 of 40 instructions a token, and these instructions more time than the
// logits' way from memory). Tokens of a node's own way join the counts for that row; mostly none lies in the quarter.
// Rows need not be aligned: loads of 16 bytes from any element on. grid: (chunks, groups of nodes, B).
// ---------------------------------------------------------------------------
template <typename T>
struct EnRun {                       // eight logits as they lie in a row
    T x[8];
} __attribute__((packed, aligned(sizeof(T))));

struct EnRulesLds {
    float x[4][EN_RULES_CHUNK / 4];
    int count[EN_RULES_CHUNK];
    unsigned short hit[4][EN_RULES_CHUNK / 4];
};

template <typename T, bool CHOOSE>
__global__ __launch_bounds__(256) void rules_kernel(EnRulesArgs a)
{
    constexpr int WAVE_TOKENS = EN_RULES_CHUNK / 4;      // 1024
    static_assert(WAVE_TOKENS == 1024, "two runs of eight a lane");
    extern __shared__ __attribute__((aligned(16))) char smem[];      // EnRulesLds, if there are penalties
    EnRulesLds &lds = *reinterpret_cast<EnRulesLds *>(smem);
    __shared__ unsigned long long s_best[EN_TREE_MAX_NODES][4];
    const int chunk = blockIdx.x, b = blockIdx.z, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int i0 = blockIdx.y * a.nodes, i1 = min(i0 + a.nodes, a.n);
    const en_token_rules &r = a.rules;

    EnTreeLane tree;
    tree.way = 0;
    unsigned long long todo = ~0ull;                     // rows to look at
    if (a.parent) {
        tree = tree_lane(a.parent + (size_t)b * a.n, a.n, EN_TREE_MAX_NODES);
        todo = __ballot(tree.present());
    }
    todo &= (i1 == 64 ? ~0ull : (1ull << i1) - 1) & ~((1ull << i0) - 1);
    if (todo == 0)
        return;
    const unsigned long long rows = todo;
    const int v0 = chunk * EN_RULES_CHUNK;
    const int w0 = v0 + wave * WAVE_TOKENS;              // the wave's tokens
    const int last = min(a.vocab - w0, WAVE_TOKENS);     // .. as many (none or fewer: <= 0)
    float rep = 1.f, freq = 0.f, pres = 0.f;
    int n_hit = 0, my_token = -1;                        // my_token: of node `lane`, in the quarter, or -1
    int *const count = lds.count + wave * WAVE_TOKENS;
    if (r.penalties_dev) {
        rep = r.penalties_dev[3 * b];
        freq = r.penalties_dev[3 * b + 1];
        pres = r.penalties_dev[3 * b + 2];
        for (int k = tid; k < EN_RULES_CHUNK; k += 256)
            lds.count[k] = 0;
        __syncthreads();
        const int h = r.history_dev ? min(max(r.history_len_dev[b], 0), r.history_stride) : 0;
        const int *const history = r.history_dev + (size_t)b * r.history_stride;
        for (int k = tid; k < h; k += 256) {
            const unsigned v = (unsigned)history[k] - (unsigned)v0;
            if (v < (unsigned)EN_RULES_CHUNK)
                atomicAdd(&lds.count[v], 1);
        }
        if (a.tokens && lane < a.n) {
            const unsigned v = (unsigned)a.tokens[(size_t)b * a.n + lane] - (unsigned)w0;
            my_token = tree.present() && (int)v >= 0 && (int)v < last ? (int)v : -1;
        }
        __syncthreads();
        for (int k = 0; k < last; k += 64) {
            const bool hit = k + lane < last && count[k + lane] > 0;
            const unsigned long long hits = __ballot(hit);
            if (hit)
                lds.hit[wave][n_hit + __popcll(hits & ((1ull << lane) - 1))] = (unsigned short)(k + lane);
            n_hit += (int)__popcll(hits);
        }
        wave_lds_order();
    }
    const unsigned long long in_quarter = __ballot(my_token >= 0);
    const float *const bias = r.bias_dev ? r.bias_dev + (size_t)b * r.bias_agent_stride : nullptr;
    const uint32_t *const mask = r.mask_dev ? r.mask_dev + (size_t)b * r.mask_agent_stride : nullptr;
    float add[2][8];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = 512 * q + 8 * lane + j;
            add[q][j] = bias && k < last ? bias[w0 + k] : 0.f;
        }

    // a lane's run q: tokens w0 + 512 q + 8 lane on
    auto load = [&](int i, T (&x)[2][8]) {
        const T *row = (const T *)a.logits + ((size_t)b * a.n + i) * a.logits_stride + w0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int k = 512 * q + 8 * lane;
            if (k + 8 <= last) {
                const EnRun<T> run = *reinterpret_cast<const EnRun<T> *>(row + k);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[q][j] = run.x[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[q][j] = k + j < last ? row[k + j] : (T)EN_NEG_INF;
            }
        }
    };
    T now[2][8], next[2][8];
    int i = __builtin_ctzll(todo);
    if (last > 0)
        load(i, now);
    while (todo && last > 0) {
        todo &= todo - 1;
        const int i_next = todo ? __builtin_ctzll(todo) : i;
        if (todo)
            load(i_next, next);
        uint32_t allowed[2] = {0xffu, 0xffu};
        if (mask) {
            const uint32_t *words = mask + (size_t)i * r.mask_node_stride;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int k = 512 * q + 8 * lane;        // (w0 and k are multiples of 8: a run's bits lie in one word)
                allowed[q] = k < last ? words[(w0 + k) >> 5] >> ((w0 + k) & 31) : 0u;
            }
        }
        float x[2][8];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[q][j] = (float)now[q][j];
        const unsigned long long way = a.parent ? readlane64(tree.way, i) : 0ull;
        const bool own = (way & in_quarter) != 0;
        if (n_hit > 0 || own) {
            float *const sx = lds.x[wave];
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    *reinterpret_cast<f32x4 *>(sx + 512 * q + 8 * lane + j) = f32x4{x[q][j], x[q][j + 1], x[q][j + 2], x[q][j + 3]};
            const bool adds = own && my_token >= 0 && (way >> lane & 1);
            bool first = false;                          // this lane takes a token that no list has
            if (adds)
                first = atomicAdd(&count[my_token], 1) == 0;
            wave_lds_order();
            for (int k = lane; k < n_hit; k += 64) {
                const int t = lds.hit[wave][k];
                sx[t] = penalised(sx[t], count[t], rep, freq, pres);
            }
            if (first)
                sx[my_token] = penalised(sx[my_token], count[my_token], rep, freq, pres);
            wave_lds_order();
            if (adds)
                atomicSub(&count[my_token], 1);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(sx + 512 * q + 8 * lane + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[q][j + e] = y[e];
                }
            wave_lds_order();
        }
        if (bias)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[q][j] += add[q][j];
        if (mask)
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[q][j] = allowed[q] >> j & 1 ? x[q][j] : EN_NEG_INF;
        if constexpr (CHOOSE) {
            float best = EN_NEG_INF;
            int token = -1;
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (x[q][j] > best) {                // (no NaN is; of equals the first stays)
                        best = x[q][j];
                        token = 512 * q + j;
                    }
            const unsigned long long w = wave_choice(token >= 0 ? rank_of(best) : 0u, w0 + token + 8 * lane);
            if (lane == 0)
                s_best[i][wave] = w;
        } else {
            T *row = (T *)a.out + ((size_t)b * a.n + i) * a.out_stride + w0;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int k = 512 * q + 8 * lane;
                EnRun<T> run;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    run.x[j] = (T)x[q][j];
                if (k + 8 <= last)
                    *reinterpret_cast<EnRun<T> *>(row + k) = run;
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (k + j < last)
                            row[k + j] = run.x[j];
            }
        }
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                now[q][j] = next[q][j];
        i = i_next;
    }
    if constexpr (CHOOSE) {
        const int waves = min(4, (a.vocab - v0 + WAVE_TOKENS - 1) / WAVE_TOKENS);    // those that had tokens
        __syncthreads();
        const int row = i0 + tid;
        if (row < i1 && (rows >> row & 1)) {
            unsigned long long best = 0;
            for (int w = 0; w < waves; ++w)
                best = s_best[row][w] > best ? s_best[row][w] : best;
            a.best[((size_t)b * a.n + row) * a.chunks + chunk] = best;
        }
    }
}

// A workgroup per agent: the choices out of their chunks' best, a wave a node, then the first wave goes down the path.
__global__ __launch_bounds__(1024) void accept_kernel(EnAcceptArgs a)
{
    __shared__ int s_choice[EN_TREE_MAX_NODES];
    const int b = blockIdx.x, lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    const size_t row = (size_t)b * a.n + lane;
    const int done = a.done[b];
    const EnTreeLane t = tree_lane(a.parent + (size_t)b * a.n, a.n, tree_room(done, a.Nq));
    int choice = -1;
    if (a.best) {
        const unsigned long long present = __ballot(t.present());
        for (int i = wave; i < a.n; i += waves) {
            unsigned long long best = 0;
            if (present >> i & 1)
                for (int c = lane; c < a.chunks; c += 64) {
                    const unsigned long long w = a.best[((size_t)b * a.n + i) * a.chunks + c];
                    best = w > best ? w : best;
                }
            const unsigned long long w = wave_choice((unsigned)(best >> 32), (int)~(unsigned)best);
            if (lane == 0)
                s_choice[i] = w ? (int)~(unsigned)w : -1;
        }
        __syncthreads();
        if (lane < a.n)
            choice = s_choice[lane];
    } else if (t.present()) {
        choice = a.choice_in[row];
    }
    if (wave != 0)
        return;
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
    const dim3 grid(a.chunks, (a.n + a.nodes - 1) / a.nodes, a.B), blk(256);
    const size_t lds = a.rules.penalties_dev ? sizeof(EnRulesLds) : 0;
    if (dtype == EN_F32)
        hipLaunchKernelGGL((rules_kernel<float, CHOOSE>), grid, blk, lds, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL((rules_kernel<bf16_t, CHOOSE>), grid, blk, lds, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
int en_launch_rules(const EnRulesArgs &a, int dtype, void *stream) { return launch_rules<false>(a, dtype, stream); }
int en_launch_choices(const EnRulesArgs &a, int dtype, void *stream) { return launch_rules<true>(a, dtype, stream); }

int en_launch_accept(const EnAcceptArgs &a, void *stream)
{
    hipLaunchKernelGGL(accept_kernel, dim3(a.B), dim3(a.best ? 64 * (a.n < 16 ? a.n : 16) : 64), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
