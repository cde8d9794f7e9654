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
// rules: a workgroup takes EN_RULES_CHUNK tokens of `a.nodes` of an agent's rows, a wave an equal share of the tokens of each
// row: 16 a lane, in two runs of eight, or one run. Reading the logits once (and writing them once) is all that choices
// without rules cost: 64 x 32 rows of 128000 tokens, bf16, 93 us, 5.6 TB/s; one agent's eight rows of 32000 3.8, which is a
// launch and two trips to memory. Under penalties the tables' set-up comes first (7 us with 2 - 4 K tokens of history), then
// the instructions a token: all rules on 16 x 13 rows of 50021 tokens 18.0 us, choices of 128000 under all rules 26.
//
// The tokens that penalties concern are few: they are counted into a table in LDS once for all rows of the workgroup, each
// wave lists those of its share, and in a row only they are divided and subtracted from, in a copy of the share in
// LDS (a division for every token would be 12 of 40 instructions a token, and these instructions more time than the
// logits' way from memory). Tokens of a node's own way join the counts for that row; mostly none lies in the share.
// Rows need not be aligned: loads of 16 bytes from any element on. grid: (groups of nodes, B, chunks): the first tokens, which
// in most vocabularies are the frequent ones, are begun first.
// ---------------------------------------------------------------------------
template <typename T>
struct EnRun {                       // eight logits as they lie in a row
    T x[8];
} __attribute__((packed, aligned(sizeof(T))));

struct EnRulesLds {
    float x[EN_RULES_CHUNK];
    int count[EN_RULES_CHUNK];
    unsigned short hit[EN_RULES_CHUNK / 4];
};

// RULES: none, a bias or a mask, or penalties too. (One instance for all rules, which keeps 128 registers and half as many waves
// where there are no penalties: choices of 64 x 32 rows of 128000 tokens under a bias and masks 161 us, so 110, of 16 x 13 18.5 /
// 17.0; 16 x 13 rows of 50021 written out 13.1 / 12.8.)
enum EnRulesKind { EN_NO_RULES, EN_FEW_RULES, EN_ALL_RULES };

// Rules that are written out take eight waves with half as many tokens each: 16 agents' 13 rows of 50021 tokens under all rules
// 19.1 us with four, 18.2 with eight, under masks 13.1 / 11.4, one row of 32000 6.1 / 5.2. Choices have a wave's exchanges for
// each row besides: 16 x 13 rows of 128000 tokens under all rules 25.8 / 27.2, under masks 16.2 / 17.6.
constexpr int en_rules_waves(bool choose, int rules) { return rules != EN_NO_RULES && !choose ? 8 : 4; }

template <typename T, bool CHOOSE, int RULES>
__global__ __launch_bounds__(64 * en_rules_waves(CHOOSE, RULES), RULES == EN_NO_RULES ? 1 : RULES == EN_ALL_RULES && CHOOSE ? 4 : 8)
void rules_kernel(EnRulesArgs a)
{
    constexpr bool RULED = RULES != EN_NO_RULES, PENALTIES = RULES == EN_ALL_RULES;
    constexpr int WAVES = en_rules_waves(CHOOSE, RULES), NT = 64 * WAVES;
    constexpr int WAVE_TOKENS = EN_RULES_CHUNK / WAVES;
    constexpr int Q = WAVE_TOKENS / 512;                 // runs of eight a lane
    constexpr int LISTED = WAVE_TOKENS / 4;              // of so many tokens that have occurred a list is worth its trips through LDS
    extern __shared__ __attribute__((aligned(16))) char smem[];      // EnRulesLds, if there are penalties
    EnRulesLds &lds = *reinterpret_cast<EnRulesLds *>(smem);
    __shared__ unsigned long long s_best[CHOOSE ? EN_TREE_MAX_NODES : 1][WAVES];
    const int chunk = blockIdx.z, b = blockIdx.y, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int i0 = blockIdx.x * a.nodes, i1 = min(i0 + a.nodes, a.n);
    const en_token_rules &r = a.rules;

    // what is asked for first, in one trip: the history's first entries (as many as there may be: how many there are is on
    // its way too), the penalties, the tree's tokens
    constexpr int HJ = 8;
    const int *const history = r.history_dev ? r.history_dev + (size_t)b * r.history_stride : nullptr;
    int early[HJ], token = -1, h = 0;
    float rep = 1.f, freq = 0.f, pres = 0.f;
    if constexpr (PENALTIES) {
        const int most = history ? r.history_stride : 0;
#pragma unroll
        for (int j = 0; j < HJ; ++j)
            early[j] = j * NT + tid < most ? history[j * NT + tid] : -1;
        if (a.tokens && lane < a.n)
            token = a.tokens[(size_t)b * a.n + lane];
        rep = r.penalties_dev[3 * b];
        freq = r.penalties_dev[3 * b + 1];
        pres = r.penalties_dev[3 * b + 2];
        h = most ? min(max(r.history_len_dev[b], 0), most) : 0;
    }

    EnTreeLane tree;
    tree.way = 0;
    unsigned long long rows = ~0ull;                     // rows to look at
    if (a.parent) {
        tree = tree_lane(tree_parent(a.parent + (size_t)b * a.n, a.n), a.n, EN_TREE_MAX_NODES);
        rows = __ballot(tree.present());
    }
    rows &= (i1 == 64 ? ~0ull : (1ull << i1) - 1) & ~((1ull << i0) - 1);
    if (rows == 0)
        return;
    const int v0 = chunk * EN_RULES_CHUNK;
    const int w0 = v0 + wave * WAVE_TOKENS;              // the wave's tokens
    const int last = min(a.vocab - w0, WAVE_TOKENS);     // .. as many (none or fewer: <= 0)
    const uint32_t *const mask = RULED && r.mask_dev ? r.mask_dev + (size_t)b * r.mask_agent_stride : nullptr;

    // a lane's run q: tokens w0 + 512 q + 8 lane on
    struct Row {
        EnRun<T> run[Q];
        uint32_t allowed[Q];
    };
    auto load = [&](int i, Row &x) __attribute__((always_inline)) {
        const T *row = (const T *)a.logits + ((size_t)b * a.n + i) * a.logits_stride + w0;
        const uint32_t *words = RULED && mask ? mask + (size_t)i * r.mask_node_stride : nullptr;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int k = 512 * q + 8 * lane;
            if (k + 8 <= last)
                x.run[q] = *reinterpret_cast<const EnRun<T> *>(row + k);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x.run[q].x[j] = k + j < last ? row[k + j] : (T)EN_NEG_INF;
            // (w0 and k are multiples of 8: a run's bits lie in one word)
            if (RULED && words)
                x.allowed[q] = k < last ? words[(w0 + k) >> 5] : 0u;
        }
    };
    unsigned long long todo = last > 0 ? rows : 0ull;
    Row now;
    if (todo)
        load(__builtin_ctzll(todo), now);

    const float *const bias = RULED && r.bias_dev ? r.bias_dev + (size_t)b * r.bias_agent_stride : nullptr;
    float add[Q][8];
    if (RULED && bias)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int k = 512 * q + 8 * lane;
            EnRun<float> run;
            if (k + 8 <= last)
                run = *reinterpret_cast<const EnRun<float> *>(bias + w0 + k);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    run.x[j] = k + j < last ? bias[w0 + k + j] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                add[q][j] = run.x[j];
        }
    int n_hit = 0, my_token = -1;                        // my_token: of node `lane`, in the share, or -1
    int *const count = lds.count + wave * WAVE_TOKENS;
    unsigned short *const hit = lds.hit + wave * LISTED;
    if constexpr (PENALTIES) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int k = 0; k < EN_RULES_CHUNK / (4 * NT); ++k)
            *reinterpret_cast<i32x4 *>(lds.count + 4 * NT * k + 4 * tid) = i32x4{0, 0, 0, 0};
        {
            const unsigned v = (unsigned)token - (unsigned)w0;
            my_token = tree.present() && token >= 0 && v < (unsigned)max(last, 0) ? (int)v : -1;
        }
        __syncthreads();
        auto counted = [&](int v, bool there) {
            if (there && (unsigned)v - (unsigned)v0 < (unsigned)EN_RULES_CHUNK)
                atomicAdd(&lds.count[v - v0], 1);
        };
#pragma unroll
        for (int j = 0; j < HJ; ++j)
            counted(early[j], j * NT + tid < h);
        for (int k0 = HJ * NT; k0 < h; k0 += HJ * NT) {
            int v[HJ];
#pragma unroll
            for (int j = 0; j < HJ; ++j)
                v[j] = k0 + j * NT + tid < h ? history[k0 + j * NT + tid] : -1;
#pragma unroll
            for (int j = 0; j < HJ; ++j)
                counted(v[j], k0 + j * NT + tid < h);
        }
        __syncthreads();
        int c[8 * Q];
#pragma unroll
        for (int k = 0; k < 8 * Q; ++k)
            c[k] = 64 * k + lane < last ? count[64 * k + lane] : 0;
#pragma unroll
        for (int k = 0; k < 8 * Q; ++k) {
            const unsigned long long hits = __ballot(c[k] > 0);
            const int at = n_hit + (int)__popcll(hits & ((1ull << lane) - 1));
            if (c[k] > 0 && at < LISTED)                 // (a longer list is not used)
                hit[at] = (unsigned short)(64 * k + lane);
            n_hit += (int)__popcll(hits);
        }
        wave_lds_order();
    }
    const unsigned long long in_share = PENALTIES ? __ballot(my_token >= 0) : 0ull;

    auto penalties = [&](float (&x)[Q][8], unsigned long long way) __attribute__((always_inline)) {
        const bool own = (way & in_share) != 0;
        if (n_hit == 0 && !own)
            return;
        const bool adds = own && my_token >= 0 && (way >> lane & 1);
        bool first = false;                              // this lane takes a token that no list has
        if (adds)
            first = atomicAdd(&count[my_token], 1) == 0;
        wave_lds_order();
        if (n_hit > LISTED) {
            // so many that every lane looks at its own tokens
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    typedef int i32x4 __attribute__((ext_vector_type(4)));
                    const i32x4 c = *reinterpret_cast<const i32x4 *>(count + 512 * q + 8 * lane + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = penalised(x[q][j + e], c[e], rep, freq, pres);
                        x[q][j + e] = c[e] > 0 ? y : x[q][j + e];
                    }
                }
        } else {
            float *const sx = lds.x + wave * WAVE_TOKENS;
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    *reinterpret_cast<f32x4 *>(sx + 512 * q + 8 * lane + j) = f32x4{x[q][j], x[q][j + 1], x[q][j + 2], x[q][j + 3]};
            wave_lds_order();
            for (int k = lane; k < n_hit; k += 64) {
                const int t = hit[k];
                sx[t] = penalised(sx[t], count[t], rep, freq, pres);
            }
            if (first)
                sx[my_token] = penalised(sx[my_token], count[my_token], rep, freq, pres);
            wave_lds_order();
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int j = 0; j < 8; j += 4) {
                    const f32x4 y = *reinterpret_cast<const f32x4 *>(sx + 512 * q + 8 * lane + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[q][j + e] = y[e];
                }
        }
        wave_lds_order();
        if (adds)
            atomicSub(&count[my_token], 1);
        wave_lds_order();
    };
    auto look_at = [&](int i, const Row &in) __attribute__((always_inline)) {
        float x[Q][8];
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[q][j] = (float)in.run[q].x[j];
        if constexpr (RULED) {
            if constexpr (PENALTIES)
                penalties(x, a.parent ? readlane64(tree.way, i) : 0ull);
            if (bias)
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[q][j] += add[q][j];
            if (mask)
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const uint32_t bits = in.allowed[q] >> (8 * lane & 31);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        x[q][j] = bits >> j & 1 ? x[q][j] : EN_NEG_INF;
                }
        }
        if constexpr (CHOOSE) {
            // The largest of each run, of the wave, the first lane that has it in its first run or else in its second, and
            // which of the run's it is: of equals the lowest token. (NaN is no maximum. A maximum passes over a quiet NaN, but
            // of a signalling one, which logits may hold as they come from memory, the hardware makes NaN: canonical numbers
            // are quiet. Without / with this, us: 64 x 32 rows of 128000 tokens 92 / 93, under a bias and masks 113 / 120, of 16 x
            // 13 under a bias and masks 17.7 / 18.5.)
            float top_of[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                top_of[q] = EN_NEG_INF;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    top_of[q] = fmaxf(top_of[q], __builtin_canonicalizef(x[q][j]));
            }
            const float top = wave_max(fmaxf(top_of[0], top_of[Q - 1]));
            const unsigned long long in0 = __ballot(top_of[0] == top), in1 = __ballot(top_of[Q - 1] == top);
            unsigned long long w = 0;
            if (top > EN_NEG_INF) {
                const int l = __builtin_ctzll(in0 ? in0 : in1);
                int at = 7;
#pragma unroll
                for (int j = 6; j >= 0; --j) {
                    const float y = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(in0 ? x[0][j] : x[Q - 1][j]), l));
                    at = y == top ? j : at;
                }
                w = (unsigned long long)rank_of(top) << 32 | (unsigned)~(w0 + (in0 ? 0 : 512) + 8 * l + at);
            }
            if (lane == 0)
                s_best[i][wave] = w;
        } else {
            T *row = (T *)a.out + ((size_t)b * a.n + i) * a.out_stride + w0;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
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
    };
    // (One row at a time: many waves with few registers hide the memory's latency better than a wave with several rows on
    // their way. Choices of 64 x 32 rows of 128000 tokens, bf16: one row 91 us, two 93, three 120, four 116, eight 151.)
    while (todo) {
        look_at(__builtin_ctzll(todo), now);
        todo &= todo - 1;
        if (todo)
            load(__builtin_ctzll(todo), now);
    }

    if constexpr (CHOOSE) {
        const int waves = min(WAVES, (a.vocab - v0 + WAVE_TOKENS - 1) / WAVE_TOKENS);    // those that had tokens
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

// accept: a workgroup per agent: the choices out of their chunks' best, a wave a node, then the first wave goes down the path,
// a ballot a node. Bound by latency: 8 nodes with 8 chunks each 2.6 us, 64 agents' 32 nodes with 32 chunks 5.0.
__global__ __launch_bounds__(1024) void accept_kernel(EnAcceptArgs a)
{
    __shared__ int s_choice[EN_TREE_MAX_NODES];
    const int b = blockIdx.x, lane = threadIdx.x % 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    const size_t row = (size_t)b * a.n + lane;
    const int done = a.done[b];
    const EnTreeLane t = tree_lane(tree_parent(a.parent + (size_t)b * a.n, a.n), a.n, tree_room(done, a.Nq));
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

template <typename T, bool CHOOSE, int RULES>
static int launch_rules_kernel(const EnRulesArgs &a, hipStream_t st)
{
    const dim3 grid((a.n + a.nodes - 1) / a.nodes, a.B, a.chunks);
    hipLaunchKernelGGL((rules_kernel<T, CHOOSE, RULES>), grid, dim3(64 * en_rules_waves(CHOOSE, RULES)),
                       RULES == EN_ALL_RULES ? sizeof(EnRulesLds) : 0, st, a);
    return (int)hipGetLastError();
}
template <typename T, bool CHOOSE>
static int launch_rules(const EnRulesArgs &a, hipStream_t st)
{
    if (a.rules.penalties_dev)
        return launch_rules_kernel<T, CHOOSE, EN_ALL_RULES>(a, st);
    return a.rules.bias_dev || a.rules.mask_dev ? launch_rules_kernel<T, CHOOSE, EN_FEW_RULES>(a, st)
                                                : launch_rules_kernel<T, CHOOSE, EN_NO_RULES>(a, st);
}
int en_launch_rules(const EnRulesArgs &a, int dtype, void *stream)
{
    return dtype == EN_F32 ? launch_rules<float, false>(a, (hipStream_t)stream) : launch_rules<bf16_t, false>(a, (hipStream_t)stream);
}
int en_launch_choices(const EnRulesArgs &a, int dtype, void *stream)
{
    return dtype == EN_F32 ? launch_rules<float, true>(a, (hipStream_t)stream) : launch_rules<bf16_t, true>(a, (hipStream_t)stream);
}

int en_launch_accept(const EnAcceptArgs &a, void *stream)
{
    hipLaunchKernelGGL(accept_kernel, dim3(a.B), dim3(a.best ? 64 * (a.n < 16 ? a.n : 16) : 64), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
