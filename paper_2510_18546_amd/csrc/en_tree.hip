// Attention over a tree of drafted tokens and the gathered context, and the accepted tokens' way into the contexts.
#include "en_tree_lane.h"

// ---------------------------------------------------------------------------
// tree_attn (bf16)
//
// All r * n rows of a KV head attend over the same L_c + done keys of the context, so the context is read once for all of
// them: 32 bytes of it per key and dimension pair against 4 D flops a row. Up to 64 rows a KV head the step is bound by
// that read, at 256 and more by the matrix instructions too. A workgroup takes up to 8 row blocks of 32 rows (a wave each)
// of a KV head and a split of its keys; 64-key tiles of K and V^T go straight into LDS, NST of them in turn, and every
// wave reads all of them there.
//
// The tree's own keys are one more tile, the last split's first: the workgroup rotates them and lays them out in LDS as a
// tile of the context would be. Its mask is a row's way, a word whose bit m is node m.
//
// S^T = K Q^T and O^T += V^T P^T with 32 x 32 x 16 products as in attn_decode_kernel: a lane's column is a query row, its
// scores of 16 keys of a 32-key block are the operand of the second product as they are (that is what the exchanged bits
// 2 and 3 of a value's column are for). Scores are in log2 units, taken against a reference that is the maximum of the
// first keys a row sees and changes only where a score is 2^59 above it. The queries, the drafted keys, the probabilities
// and the output are rounded to bf16 once each (what the products take); sums, references and what the splits leave for
// the merge are float32.
//
// 16-byte chunks of a row lie in LDS exchanged by XOR with its number, so that 16 consecutive rows' reads of the same
// chunk meet distinct banks; the loads bring them there by reading their source in that order.
// ---------------------------------------------------------------------------
// Values that may be infinite or NaN are looked at, left out and added as bits: this library is built without NaN compares,
// and a NaN may be taken not to occur wherever a floating-point operation sees it.
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bool no_number(unsigned short bf16) { return (bf16 & 0x7f80) == 0x7f80; }

// KW = 2: two waves share a row block, a 32-key block of every tile each, and meet at the end.
template <int D, int RW, int KW, int NST>
__global__ __launch_bounds__(64 * RW * KW, RW * KW == 2 ? 1 : 2) void tree_attn_kernel(EnTreeArgs a)
{
    constexpr int W = RW * KW;
    constexpr int NT = 64 * W;                   // threads
    constexpr int KB = 32;                       // keys per matrix-instruction block
    constexpr int LB = EN_KEY_TILE;              // keys per tile
    constexpr int NUW = LB / KB / KW;            // blocks of a tile per wave
    constexpr int NKS = D / 16;
    constexpr int NDB = D / 32;
    constexpr int ROWB = 2 * D;                  // bytes per K row
    constexpr int KBYTES = LB * ROWB;
    constexpr int VROWB = 2 * LB;                // bytes per V^T row of a tile
    constexpr int VBYTES = D * VROWB;
    constexpr int STAGE = KBYTES + VBYTES;
    constexpr int NBK = KBYTES / 1024, NBV = VBYTES / 1024;      // loader blocks
    constexpr int PER = (NBK + NBV) / W;         // loads per wave and tile
    static_assert(NBK % W == 0 && NBV % W == 0 && NST >= 2, "whole loader blocks per wave");
    __shared__ __attribute__((aligned(1024))) char smem[NST * STAGE];
    __shared__ int s_no_number;                  // a value of the tree is infinite or NaN
    typedef __bf16 pair_t __attribute__((ext_vector_type(2)));

    // Neighbours in this order share a split's keys, and an XCD takes a run of them.
    const unsigned per_xcd = gridDim.x / EN_XCDS;
    const unsigned unit = (blockIdx.x % EN_XCDS) * per_xcd + blockIdx.x / EN_XCDS;
    if (unit >= a.n_units)
        return;
    unsigned t = divided(unit, a.by_ptiles);
    const int ptile = unit - t * a.n_ptiles;
    unsigned t2 = divided(t, a.by_splits);
    const int sp = a.n_splits - 1 - (t - t2 * a.n_splits);       // the last split, which has the tree, starts first
    const int b = divided(t2, a.by_hkv);
    const int kvh = t2 - b * a.Hkv;

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int lane = tid % 64;
    const int col = lane % 32, half = lane / 32;
    const int rw = wave % RW, kw = wave / RW;
    const int r = a.Hq / a.Hkv, n = a.n;
    const int n_rows = r * n;
    const int c_row = (ptile * RW + rw) * 32 + col;
    const bool row_there = c_row < n_rows;
    const int hl = row_there ? divided(c_row, a.by_n) : 0;
    const int i_row = row_there ? c_row - hl * n : 0;
    const int hq = kvh * r + hl;

    const int done = as_table(a.done)[b];
    const int Lc = as_table(a.hdr)[4 * b + 1];
    const EnTreeLane tree = tree_lane(a.parent + (size_t)b * n, n, tree_room(done, a.Nq));
    const unsigned long long present = __ballot(tree.present());
    const unsigned rows_all = (unsigned)a.B * a.Hq * n;
    const unsigned row = ((unsigned)b * a.Hq + hq) * n + i_row;
    const int L = Lc + done;                     // keys of the context (an idle agent's is not used)
    const int n_ctx = present ? (L + LB - 1) / LB : 0;
    const int t_begin = split_first_tile(sp, n_ctx + 1, a.n_splits);
    const int t_end = min((int)split_first_tile(sp + 1, n_ctx + 1, a.n_splits), n_ctx);
    const bool has_tree = sp == a.n_splits - 1 && present;
    const int n_it = max(t_end - t_begin, 0) + (has_tree ? 1 : 0);
    if (n_it == 0) {
        // nothing to do: an idle agent, or one with fewer tiles than splits
        if (row_there && half == 0 && kw == 0) {
            if (a.n_splits > 1) {
                f32x2 none = {EN_NEG_INF, 0.f};
                *reinterpret_cast<f32x2 *>(a.ws_ml + ((size_t)sp * rows_all + row) * 2) = none;
            } else {
                bf16_t *op = (bf16_t *)a.out + (((size_t)b * n + i_row) * a.Hq + hq) * D;
                for (int d = 0; d < D; d += 8)
                    *reinterpret_cast<bf16x8 *>(op + d) = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
        }
        return;
    }

    // ---- loader ----
    const char *kg = (const char *)a.kc + ((size_t)b * a.Hkv + kvh) * (size_t)a.T * ROWB;
    const char *vg = (const char *)a.vt + ((size_t)b * a.Hkv + kvh) * (size_t)a.T * ROWB;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    // chunk c of K row `row` lies at c ^ k_pattern(row), chunk c of V^T row d at c ^ v_pattern(d)
    auto k_pattern = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
    auto v_pattern = [](int d) { return (d >> 1) & 7; };
    uint32_t koff[NBK / W], voff[NBV / W];
#pragma unroll
    for (int j = 0; j < NBK / W; ++j) {
        const int q = (wave + W * j) * 64 + lane;
        const int krow = q / (ROWB / 16);
        koff[j] = (uint32_t)(krow * ROWB + ((q % (ROWB / 16)) ^ k_pattern(krow)) * 16);
    }
#pragma unroll
    for (int j = 0; j < NBV / W; ++j) {
        const int q = (wave + W * j) * 64 + lane;
        const int d = q / 8;
        voff[j] = (uint32_t)d * (uint32_t)a.T * 2u + (uint32_t)(((q % 8) ^ v_pattern(d)) * 16);
    }
    auto issue = [&](int tile, int stage) {
        const char *kt = kg + (size_t)tile * KBYTES;
        const char *vtile = vg + (size_t)tile * VROWB;
        const uint32_t dst = lds0 + stage * STAGE + wave * 1024;
#pragma unroll
        for (int j = 0; j < NBK / W; ++j)
            dma16(kt, koff[j], dst + W * j * 1024);
#pragma unroll
        for (int j = 0; j < NBV / W; ++j)
            dma16(vtile, voff[j], dst + KBYTES + W * j * 1024);
    };
    const int ctx0 = t_begin - (has_tree ? 1 : 0);       // iteration it takes tile ctx0 + it of the context
#pragma unroll
    for (int it = 0; it < NST - 1; ++it)
        if (it < n_it && !(has_tree && it == 0))
            issue(ctx0 + it, it);

    // ---- Q: load, rotate at the node's position, scale, round to bf16 ----
    const unsigned long long way = __shfl(tree.way, i_row, 64);
    const int depth = __shfl(tree.depth, i_row, 64);
    const bool row_valid = row_there && way != 0;
    bf16x8 qf[NKS];
    if (row_valid) {
        const bf16_t *qp = (const bf16_t *)a.q + (((size_t)b * n + i_row) * a.Hq + hq) * D + 8 * half;
        const size_t pos = L + depth;
        const float *ct = a.cos_tab + pos * (D / 2) + 8 * half, *st = a.sin_tab + pos * (D / 2) + 8 * half;
        bf16x8 qraw[NKS];
        f32x8 cs[NKS / 2], sn[NKS / 2];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
            qraw[ks] = *reinterpret_cast<const bf16x8 *>(qp + 16 * ks);
#pragma unroll
        for (int ks = 0; ks < NKS / 2; ++ks) {
            cs[ks] = *reinterpret_cast<const f32x8 *>(ct + 16 * ks);
            sn[ks] = *reinterpret_cast<const f32x8 *>(st + 16 * ks);
        }
#pragma unroll
        for (int ks = 0; ks < NKS / 2; ++ks)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y1, y2;
                rope_scale_pair((float)qraw[ks][j], (float)qraw[ks + NKS / 2][j], cs[ks][j], sn[ks][j], a.scale_log2e, y1, y2);
                qf[ks][j] = (bf16_t)y1;
                qf[ks + NKS / 2][j] = (bf16_t)y2;
            }
    } else {
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
            qf[ks] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
    }

    // ---- the tree's tile into stage 0 ----
    if (has_tree) {
        if (tid == 0)
            s_no_number = 0;
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        constexpr int PAIRS = D / 16;            // 8 dimensions and their partners
        bool odd = false;
        for (int x = tid; x < LB * PAIRS; x += NT) {
            const int m = x / PAIRS, c = x % PAIRS;
            const int d_m = __popcll(__shfl(tree.way, m, 64)) - 1;       // (the loop's lanes go together: NT divides)
            const bool there = present >> m & 1;
            bf16x8 k1 = {0, 0, 0, 0, 0, 0, 0, 0}, k2 = k1;
            u16x8 v1 = {0, 0, 0, 0, 0, 0, 0, 0}, v2 = v1;
            if (there) {
                const size_t from = (((size_t)b * n + m) * a.Hkv + kvh) * D + 8 * c;
                const bf16_t *kr = (const bf16_t *)a.k_rows + from, *vr = (const bf16_t *)a.v_rows + from;
                const size_t at = (size_t)(L + d_m) * (D / 2) + 8 * c;
                const f32x8 cs = *reinterpret_cast<const f32x8 *>(a.cos_tab + at), sn = *reinterpret_cast<const f32x8 *>(a.sin_tab + at);
                k1 = *reinterpret_cast<const bf16x8 *>(kr);
                k2 = *reinterpret_cast<const bf16x8 *>(kr + D / 2);
                v1 = *reinterpret_cast<const u16x8 *>(vr);
                v2 = *reinterpret_cast<const u16x8 *>(vr + D / 2);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float y1, y2;
                    rope_key_pair((float)k1[j], (float)k2[j], cs[j], sn[j], y1, y2);
                    k1[j] = (bf16_t)y1;
                    k2[j] = (bf16_t)y2;
                    // no number has no place in a product with weights of 0: it joins the sums of the rows that see it
                    // behind the loop
                    const bool n1 = no_number(v1[j]), n2 = no_number(v2[j]);
                    odd = odd || n1 || n2;
                    v1[j] = n1 ? 0 : v1[j];
                    v2[j] = n2 ? 0 : v2[j];
                }
            }
            const int pat = k_pattern(m);
            *reinterpret_cast<bf16x8 *>(smem + m * ROWB + (c ^ pat) * 16) = k1;
            *reinterpret_cast<bf16x8 *>(smem + m * ROWB + ((c + PAIRS) ^ pat) * 16) = k2;
            const int vc = (m & ~0xC) | ((m & 4) << 1) | ((m & 8) >> 1);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                auto put = [&](int d, unsigned short v) {
                    *reinterpret_cast<unsigned short *>(smem + KBYTES + d * VROWB + ((vc / 8) ^ v_pattern(d)) * 16 + vc % 8 * 2) = v;
                };
                put(8 * c + j, v1[j]);
                put(8 * c + j + D / 2, v2[j]);
            }
        }
        if (__any(odd) && lane == 0)
            s_no_number = 1;
    }

    // ---- state ----
    f32x16 o[NDB];
#pragma unroll
    for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            o[d][e] = 0.f;
    float m_ref = 0.f, l = 0.f;                  // l: this lane's share
    f32x16 negm;                                 // -m_ref
#pragma unroll
    for (int e = 0; e < 16; ++e)
        negm[e] = 0.f;
    bool has_ref = !row_valid;                   // (rows that are not there need none)
    const int kpat = D == 128 ? col & 15 : (col >> 1) & 7, vpat = (col >> 1) & 7;
    const int u0 = kw * NUW;

    for (int it = 0; it < n_it; ++it) {
        const int stage = it % NST;
        const char *stg = smem + stage * STAGE;
        // this tile's loads have landed when at most those of the later tiles are outstanding; all of them near the end
        if (it + NST - 2 < n_it)
            __builtin_amdgcn_s_waitcnt((((NST - 2) * PER) & 15) | ((((NST - 2) * PER) >> 4) << 14) | 0x0f70);
        else
            __builtin_amdgcn_s_waitcnt(0x0f70);
        __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0): the previous tile has been read, the tree's written
        __builtin_amdgcn_s_barrier();
        if (it + NST - 1 < n_it)
            issue(ctx0 + it + NST - 1, (it + NST - 1) % NST);
        lds_data_ready();
        const bool is_tree = has_tree && it == 0;
        const int kb = (ctx0 + it) * LB;         // first key of a context tile
        const int left = L - kb;                 // keys of a context tile from its first on
        if (!is_tree && left < LB) {
            // columns behind the context's last token become zero: whatever they hold has no weight, but 0 times infinity
            // is no 0
            for (int x = tid; x < D * 8; x += NT) {
                char *at = smem + stage * STAGE + KBYTES + x * 16;
                const int c = (x % 8) ^ v_pattern(x / 8);        // its chunk: columns 8 c .. 8 c + 7
                const int key = 16 * (c / 2) + 4 * (c % 2);      // .. which are these keys, 0 .. 3 and 8 .. 11 on from it
                u16x8 v = *reinterpret_cast<const u16x8 *>(at);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    v[j] = key + 8 * (j / 4) + j % 4 < left ? v[j] : 0;
                *reinterpret_cast<u16x8 *>(at) = v;
            }
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_s_barrier();
            lds_data_ready();
        }
        // ---- S^T = K Q^T - m_ref ----
        f32x16 sv[NUW];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int u = 0; u < NUW; ++u) {
                const bf16x8 fr = *reinterpret_cast<const bf16x8 *>(stg + ((u0 + u) * KB + col) * ROWB + ((2 * ks + half) ^ kpat) * 16);
                sv[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, qf[ks], ks == 0 ? negm : sv[u], 0, 0, 0);
            }
        // Hidden keys: element e of block u is key 32 u + 8 (e / 4) + e % 4 + 4 half of the tile. (Masks by arithmetic:
        // as comparisons they would take two scalar registers each.)
        if (is_tree || left < LB) {
            const unsigned long long keys = is_tree ? way : (1ull << left) - 1;
#pragma unroll
            for (int u = 0; u < NUW; ++u) {
                const uint32_t sees = (uint32_t)(keys >> (KB * (u0 + u))) >> (4 * half);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t on = (uint32_t)((int32_t)(sees << (31 - (8 * (e / 4) + e % 4))) >> 31);
                    sv[u][e] = __uint_as_float((__float_as_uint(sv[u][e]) & on) | (0xff800000u & ~on));
                }
            }
        }
        // ---- a reference for rows that have none or whose scores have outgrown it ----
        float mx = sv[0][0];
#pragma unroll
        for (int u = 0; u < NUW; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                mx = fmaxf(mx, sv[u][e]);
        if (__any(!has_ref || mx > 59.f)) {
            mx = pair_max(mx);
            const bool fix = (!has_ref || mx > 59.f) && mx > EN_NEG_INF;
            const float delta = fix ? mx : 0.f;
            const float alpha = fix ? (has_ref ? fast_exp2(-delta) : 0.f) : 1.f;
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    o[d][e] *= alpha;
            l *= alpha;
            has_ref = has_ref || fix;
            m_ref += delta;
#pragma unroll
            for (int e = 0; e < 16; ++e)
                negm[e] = -m_ref;
#pragma unroll
            for (int u = 0; u < NUW; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    sv[u][e] -= delta;
        }
        // ---- probabilities; the sums use the rounded ones, like the products ----
        bf16x8 pf[NUW][2];
#pragma unroll
        for (int u = 0; u < NUW; ++u)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const pair_t pb = {(bf16_t)fast_exp2(sv[u][e]), (bf16_t)fast_exp2(sv[u][e + 1])};
                pf[u][e / 8][e % 8] = pb[0];
                pf[u][e / 8][e % 8 + 1] = pb[1];
                l = __builtin_amdgcn_fdot2_f32_bf16(pb, pair_t{(bf16_t)1.f, (bf16_t)1.f}, l, false);
            }
        // ---- O^T += V^T P^T ----
#pragma unroll
        for (int u = 0; u < NUW; ++u)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int d = 0; d < NDB; ++d) {
                    const bf16x8 v = *reinterpret_cast<const bf16x8 *>(stg + KBYTES + (32 * d + col) * VROWB +
                                                                       ((4 * (u0 + u) + 2 * kk + half) ^ vpat) * 16);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[u][kk], o[d], 0, 0, 0);
                }
    }

    l += xor32(l);
    // ---- two waves of a row block meet: the second leaves its state in LDS, the first takes it up ----
    if constexpr (KW == 2) {
        __builtin_amdgcn_s_waitcnt(0xc07f);
        __builtin_amdgcn_s_barrier();            // everybody is done with the tiles
        lds_data_ready();
        // [row block][register][lane], four registers at a time
        f32x4 *so = reinterpret_cast<f32x4 *>(smem) + rw * (NDB * 4 + 1) * 64;
        static_assert(RW * (NDB * 4 + 1) * 1024 <= NST * STAGE, "the waves' sums fit the stages");
        if (kw == 1) {
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    so[(4 * d + g) * 64 + lane] = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
            so[NDB * 4 * 64 + lane] = f32x4{m_ref, l, 0.f, 0.f};
        }
        __syncthreads();
        if (kw == 1)
            return;
        const f32x4 other = so[NDB * 4 * 64 + lane];
        // (a sum is 0 where the wave had no key that the row sees, by the bits: one of NaN is not)
        const bool mine = __float_as_uint(l) != 0u, its = __float_as_uint(other[1]) != 0u;
        const float m = mine && its ? fmaxf(m_ref, other[0]) : mine ? m_ref : other[0];
        const float wm = mine ? fast_exp2(m_ref - m) : 0.f, wo = its ? fast_exp2(other[0] - m) : 0.f;
        l = (mine ? l * wm : 0.f) + (its ? other[1] * wo : 0.f);
        m_ref = m;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 x = so[(4 * d + g) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[d][4 * g + e] = (mine ? o[d][4 * g + e] * wm : 0.f) + (its ? x[e] * wo : 0.f);
            }
    }
    if (!row_there)
        return;
    if (!row_valid)
        l = 0.f;
    if (has_tree && s_no_number) {
        // what the tree's tile left out: infinite with any weight, or NaN
#pragma unroll 1
        for (int m = 0; m < n; ++m) {
            const bf16_t *vr = (const bf16_t *)a.v_rows + (((size_t)b * n + m) * a.Hkv + kvh) * D + 4 * half;
            if (way >> m & 1)
#pragma unroll
                for (int d = 0; d < NDB; ++d)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const u16x4 v = *reinterpret_cast<const u16x4 *>(vr + 32 * d + 8 * g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[d][4 * g + e] += __uint_as_float(no_number(v[e]) ? (uint32_t)v[e] << 16 : 0u);
                    }
        }
    }
    if (a.n_splits > 1) {
        const size_t part = (size_t)sp * rows_all + row;
        if (half == 0) {
            f32x2 v = {m_ref, l};
            *reinterpret_cast<f32x2 *>(a.ws_ml + part * 2) = v;
        }
        if (!row_valid)
            return;                              // (a sum of 0: nobody reads the rest)
        float *op = a.ws_opart + part * D + 4 * half;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(op + 32 * d + 8 * g) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    } else {
        const float inv = row_valid ? 1.f / l : 0.f;
        bf16_t *op = (bf16_t *)a.out + (((size_t)b * n + i_row) * a.Hq + hq) * D + 4 * half;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = row_valid ? (bf16_t)(o[d][4 * g + e] * inv) : (bf16_t)0.f;
                *reinterpret_cast<bf16x4 *>(op + 32 * d + 8 * g) = v;
            }
    }
}

// ---------------------------------------------------------------------------
// tree_merge: out = sum_sp 2^(m_sp - m) O_sp / sum_sp 2^(m_sp - m) l_sp. A thread takes four values of a row, neighbours the
// row's next four, and G groups of D / 4 threads share the splits of a row and meet in LDS. A split that a row saw nothing
// of left a sum of 0 and no values; a row without any is zero. grid: rows * G * (D / 4) threads.
// ---------------------------------------------------------------------------
template <typename T, int D, int G>
__global__ __launch_bounds__(256) void tree_merge_kernel(EnTreeArgs a)
{
    constexpr int CH = D / 4, RPW = 256 / (CH * G);      // threads per group; rows per workgroup
    static_assert(RPW >= 1, "a row's groups are in a workgroup");
    __shared__ f32x4 s_acc[G > 1 ? 256 : 1];
    __shared__ f32x2 s_ml[G > 1 ? 256 : 1];
    const unsigned rows = (unsigned)a.B * a.Hq * a.n;
    const int tid = threadIdx.x, ch = tid % CH, g = tid / CH % G;
    const unsigned row = blockIdx.x * RPW + tid / (CH * G);
    constexpr int NB = G == 1 ? 8 : 4;
    float M = EN_NEG_INF, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (row < rows)
        for (int sp0 = g; sp0 < a.n_splits; sp0 += NB * G) {
            f32x2 ml[NB];
            f32x4 v[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const bool on = sp0 + j * G < a.n_splits;
                const size_t part = (size_t)(on ? sp0 + j * G : sp0) * rows + row;
                ml[j] = *reinterpret_cast<const f32x2 *>(a.ws_ml + part * 2);
                v[j] = *reinterpret_cast<const f32x4 *>(a.ws_opart + part * D + 4 * ch);
                if (!on)
                    ml[j][1] = 0.f;
            }
            float Mb = M;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                Mb = __float_as_uint(ml[j][1]) ? fmaxf(Mb, ml[j][0]) : Mb;
            const float keep = M == EN_NEG_INF ? 0.f : fast_exp2(M - Mb);
            l *= keep;
            acc *= keep;
            M = Mb;
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (__float_as_uint(ml[j][1])) {
                    const float w = fast_exp2(ml[j][0] - M);
                    l += w * ml[j][1];
                    acc += w * v[j];
                }
        }
    if constexpr (G > 1) {
        s_acc[tid] = acc;
        s_ml[tid] = f32x2{M, l};
        __syncthreads();
        if (g != 0)
            return;
        f32x2 ml[G];
#pragma unroll
        for (int k = 0; k < G; ++k) {
            ml[k] = s_ml[tid + k * CH];
            M = __float_as_uint(ml[k][1]) ? fmaxf(M, ml[k][0]) : M;
        }
        l = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < G; ++k)
            if (__float_as_uint(ml[k][1])) {
                const float w = fast_exp2(ml[k][0] - M);
                l += w * ml[k][1];
                acc += w * s_acc[tid + k * CH];
            }
    }
    if (row >= rows)
        return;
    const float inv = __float_as_uint(l) ? 1.f / l : 0.f;
    const unsigned bh = divided(row, a.by_n), i = row - bh * a.n;
    const unsigned b = divided(bh, a.by_hq), hq = bh - b * a.Hq;
    typedef T tvec __attribute__((ext_vector_type(4)));
    *reinterpret_cast<tvec *>((T *)a.out + (((size_t)b * a.n + i) * a.Hq + hq) * D + 4 * ch) = __builtin_convertvector(acc * inv, tvec);
}

template <typename T, int D>
static void launch_merge(const EnTreeArgs &a, hipStream_t st)
{
    const unsigned rows = (unsigned)a.B * a.Hq * a.n;
    const auto grid = [rows](int G) { return dim3((rows + 1024 / (D * G) - 1) / (1024 / (D * G))); };
    if (a.n_splits > 8 && rows < 2048)
        hipLaunchKernelGGL((tree_merge_kernel<T, D, 8>), grid(8), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((tree_merge_kernel<T, D, 1>), grid(1), dim3(256), 0, st, a);
}

template <int D>
static int launch_tree_bf16(const EnTreeArgs &a, int blocks, hipStream_t st)
{
    const dim3 grid((a.n_units + EN_XCDS - 1) / EN_XCDS * EN_XCDS);
    if (blocks == 1)
        hipLaunchKernelGGL((tree_attn_kernel<D, 1, 2, 2>), grid, dim3(128), 0, st, a);
    else if (blocks == 2)
        hipLaunchKernelGGL((tree_attn_kernel<D, 2, 2, 2>), grid, dim3(256), 0, st, a);
    else if (blocks == 4)
        hipLaunchKernelGGL((tree_attn_kernel<D, 4, 1, 2>), grid, dim3(256), 0, st, a);
    else if (blocks == 8)
        hipLaunchKernelGGL((tree_attn_kernel<D, 8, 1, 4>), grid, dim3(512), 0, st, a);
    else
        return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}
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

int en_launch_tree_attention(const en_pool *pool, const EnTreeArgs &a, int blocks, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const int D = pool->d.head_dim;
    if (pool->d.dtype != EN_F32)
        return D == 64 ? launch_tree_bf16<64>(a, blocks, st) : launch_tree_bf16<128>(a, blocks, st);
    const dim3 grid(a.n, a.Hq, a.B), blk(256);
    if (D == 64)
        hipLaunchKernelGGL((tree_attention_kernel<float, 64>), grid, blk, 0, st, a);
    else
        hipLaunchKernelGGL((tree_attention_kernel<float, 128>), grid, blk, 0, st, a);
    return (int)hipGetLastError();
}

int en_launch_tree_merge(const en_pool *pool, const EnTreeArgs &a, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    if (pool->d.dtype == EN_F32) {
        if (pool->d.head_dim == 64)
            launch_merge<float, 64>(a, st);
        else
            launch_merge<float, 128>(a, st);
    } else {
        if (pool->d.head_dim == 64)
            launch_merge<bf16_t, 64>(a, st);
        else
            launch_merge<bf16_t, 128>(a, st);
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
