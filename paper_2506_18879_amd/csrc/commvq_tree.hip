// Attention of drafted tokens (trees of up to 64 nodes per sequence) over a paged compressed cache.
//
// Row r of (sequence b, KV head g) is query head g G + r % G of node r / G; the rows of a KV head share its decoded keys and values.
// With t0 the position of a sequence's first node, a row's logit with a cached token at position p is
//     (q R_t) . (k R_p) scale = Re( [q conj E(t - t0)] conj[k conj E(p - t0)] ) scale,   E(m) = exp(i m theta_j) in sub-space j,
// so that both sides are turned once, by distances that the phase tables cover, and everything after that is a dense product:
// logits K Q^T, weights exp(logit - max), and weights times V, with the running maximum and sum of a softmax.  A range of a context's tokens
// leaves an unnormalised row, its maximum and its sum; k_tree_final joins the ranges with the node's own part.
#include "commvq_internal.hpp"

#include <algorithm>

commvq_status commvq_check_pages(const commvq_pages *p);

namespace {

constexpr int kMaxNodes = 64;
constexpr int kChunk = 32;            // tokens that a workgroup of k_tree_rows decodes at a time: one k-step of the second product
constexpr int kRowBytes = 2 * kD + 16;  // decoded rows in LDS: 16 bytes apart in the banks, for reads of 16 rows at one place
constexpr int kWideChunk = 16;        // tokens of a chunk of k_tree_rows_f32
constexpr int kWideRow = kD + 4;      // its rows in LDS, in floats

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));

struct TreeArgs {
    const void *q, *node_k, *node_v;
    const uint8_t *key_pages, *val_pages;
    const void *key_cb, *val_cb;
    const int32_t *seq_lens, *tables, *cu, *node_pos, *key_pos;
    const unsigned long long *mask;
    const float2 *tbl_hi, *tbl_lo;
    float *part;                      // [row][splits][d] unnormalised
    float2 *stat;                     // [row][splits] (maximum in powers of 2, sum)
    void *out;
    const float *scales;              // [head] (keys', values' power of two), behind the streamed codebooks
    unsigned axes[4];                 // axis of sub-space j: bits 2 (j % 16) of word j / 16
    long long q_stride, node_stride;
    int batch, Hq, Hkv, G, Mk, Mv, n_hi, n_axes;
    int block_bits, n_blocks, max_blocks;
    int total_nodes, max_nodes, max_seqlen;
    int splits, split_len, row_tiles;
    int halves;                       // parts of a range of split_len tokens
    int turn;                         // 0: position_free, nothing is turned
    int q_bf16, cb_bf16;
    float scale2;                     // softmax scale times log2(e)
};

// Sequence b's tokens and nodes, whatever the device arrays hold: inside the buffers that the host has described.
struct Span {
    int L, n0, n;
};
__device__ __forceinline__ Span span_of(const TreeArgs &a, int b)
{
    Span s;
    s.L = min(max(a.seq_lens[b], 0), a.max_seqlen);
    s.n0 = min(max(a.cu[b], 0), a.total_nodes);
    s.n = min(min(max(a.cu[b + 1], s.n0), a.total_nodes) - s.n0, a.max_nodes);
    return s;
}
__device__ __forceinline__ int axis_of(const TreeArgs &a, int j)
{
    // (no indexing by lane: the words would be put into memory, or LDS, for it)
    const unsigned w = j & 32 ? (j & 16 ? a.axes[3] : a.axes[2]) : (j & 16 ? a.axes[1] : a.axes[0]);
    return (int)(w >> (2 * (j & 15))) & 3;
}

// E(m) of sub-space j, conjugated where `back` says so: a vector z turned by R_m is z conj E(m)
__device__ __forceinline__ float2 turned_by(const TreeArgs &a, int m, int j)
{
    const unsigned d = m < 0 ? 0u - (unsigned)m : (unsigned)m;
    const float2 h = a.tbl_hi[(size_t)min(d >> kLoBits, (unsigned)(a.n_hi - 1)) * kJ + j], l = a.tbl_lo[(size_t)(d & (kLo - 1)) * kJ + j];
    const float x = h.x * l.x - h.y * l.y, y = h.x * l.y + h.y * l.x;
    return make_float2(x, m < 0 ? y : -y);       // conj E(m)
}
__device__ __forceinline__ float2 times(float2 a, float2 b) { return make_float2(a.x * b.x - a.y * b.y, a.x * b.y + a.y * b.x); }

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    const bf16x2_t p = __builtin_convertvector(f2{lo, hi}, bf16x2_t);  // to nearest, ties to even
    return __builtin_bit_cast(unsigned, p);
}

// Two fp32 numbers as two bf16 parts each: what is nearest, and what is left of it.  (Of an infinity nothing is left, not a NaN.)
__device__ __forceinline__ uint2_t split_bf16(float lo, float hi)
{
    const unsigned top = pack_bf16(lo, hi);
    const float x = lo - bf16_lo(top), y = hi - bf16_hi(top);
    return uint2_t{top, pack_bf16(x == x ? x : 0.f, y == y ? y : 0.f)};
}
// acc + (a + al)(b + bl), without the product of the small parts
__device__ __forceinline__ floatx4_t product(uint4_t a, uint4_t al, uint4_t b, uint4_t bl, floatx4_t acc)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, al), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, bl), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}

// The maximum over lanes l, l ^ 16, l ^ 32 and l ^ 48.
__device__ __forceinline__ float quads_max(float v)
{
    const unsigned u = __builtin_bit_cast(unsigned, v);
    auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned a0 = a[0], a1 = a[1], w = __builtin_bit_cast(unsigned, fmaxf(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const unsigned b0 = b[0], b1 = b[1];
    return fmaxf(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}

// fp16 pairs: what the kernels of long contexts keep keys, values, queries and weights in.  Eleven bits instead of bf16's eight; the range is seen to
// by powers of two, for keys and values one each per head (the codebooks': see k_tree_scale), for queries one per row
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
__device__ __forceinline__ unsigned pack_f16(float lo, float hi)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f2{lo, hi}, f16x2_t));  // to nearest, ties to even
}
// the power of two that brings the largest of a row's elements to 2^9 .. 2^10 (1 if there is none, or one that is not finite)
__device__ __forceinline__ float half_scale(float top)
{
    if (!(top > 0.f && top < INFINITY)) return 1.f;
    int e;
    (void)frexpf(top, &e);
    return ldexpf(1.f, min(max(10 - e, -100), 100));
}

// 16-bit elements of column l % 16 out of a 4 x 16 block of rows that the 16 lanes around l point at, 8 bytes each, row by row
typedef __attribute__((address_space(3))) short4_t *lds_s4_ptr;
__device__ __forceinline__ uint2_t lds_read_columns(const void *p)
{
    const short4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(p));
    return __builtin_bit_cast(uint2_t, v);
}

// first operand of the gather sums (see k_score_stream): rows 0..7 add element i of the four lanes' first pieces, rows 8..15 of their second
__device__ __forceinline__ void selection(int lane, uint4_t &sel, unsigned &sidx)
{
    const int n = lane & 15, gk = lane >> 4, e = n & 7, t = e >> 2, pos = e & 3, other = pos == 0 ? 1 : 0;
    sel = uint4_t{0u, 0u, 0u, 0u};
    sidx = 0x44444444u;
    if ((n < 8) == (gk < 2)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((i & 1) == t) sel[i] = 0x00003f80u;
        const unsigned pair = (unsigned)pos | (unsigned)other << 2;
        sidx = (sidx & ~(0xfu << (4 * t)) & ~(0xfu << (4 * (2 + t)))) | pair << (4 * t) | pair << (4 * (2 + t));
        sidx = (sidx & 0xffffu) | sidx << 16;
    }
}

// ------------------------------------------------------------------ k_tree_rows
// One range of a context for NR tiles of 16 rows of a KV head, 32 tokens at a time.  All eight wavefronts decode four tokens of them each; then
// 8 / NR of them have a row tile, and different elements of it (whose logits each makes by itself).
// Decode: the four 16-lane rows of a wavefront hold four codebooks, a lane a 16-byte piece of a codeword; two tokens' pieces
// are the dense operand of v_smfmac_f32_16x16x64_bf16, whose constant 0/1 operand adds them in fp32 (exactly: products with 1.0).
// A lane then has four elements of one token, turns them (keys), splits each into two bf16 parts (16 bits; the codebooks' range needs bf16's, and
// one part alone costs a few hundred tokens' result 2^-9 more than its own rounding) and leaves them in LDS.  Queries and weights likewise; of a
// product's four parts the three that count are added.  Products: K Q^T with tokens as rows, so that a lane has 4 tokens of one query row; what it
// makes of them is, without any exchange, the operand of V^T P^T, whose other operand is read from LDS by columns.
// Short contexts are bound by the chain pages -> codes -> rows, so codes are asked for a chunk ahead and a wavefront's rows all at once; longer
// ones by the codeword rows' way through the L1s, 256 bytes a codebook and token.  Measured: 8 heads, 32 rows each, 701 tokens, 32 codebooks 17.2 us.
constexpr int kRowsWaves = 8;
constexpr int kOwn = kChunk / kRowsWaves;       // tokens that a wavefront decodes of a chunk
template <int NR, bool AXES>
__global__ __launch_bounds__(64 * kRowsWaves) void k_tree_rows(const TreeArgs a)
{
    constexpr int ND = kRowsWaves / NR, NX = 8 / ND;                 // wavefronts of a row tile; tiles of 16 elements of a wavefront
    __shared__ __align__(16) char ktile[2][kChunk * kRowBytes], vtile[2][kChunk * kRowBytes];   // high and low parts
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int id = blockIdx.x;
    const int g = id % a.Hkv;
    id /= a.Hkv;
    const int rt = id % a.row_tiles;
    id /= a.row_tiles;
    const int split = id % a.splits, b = id / a.splits;
    const Span s = span_of(a, b);
    const int R = s.n * a.G, r0 = rt * 16 * NR, t_begin = split * a.split_len, t_end = min(s.L, t_begin + a.split_len);
    if (r0 >= R || t_begin >= t_end) return;
    const int n = lane & 15, gk = lane >> 4, wr = wave / ND, wd = wave % ND;

    // codes of the wavefront's tokens c0 + 4 wave .. + 3, a chunk ahead: lane row gk has books 4 gk .. + 3 of every block of 16
    const int32_t *table = a.tables + (size_t)b * a.max_blocks;
    const int in_page = (1 << a.block_bits) - 1;
    unsigned seen_next = 0, ck_next[kOwn][2], cv_next[kOwn][2];
    int slot_next = 0;                                               // of token c0 + lane % 32
    auto ask = [&](int c0) __attribute__((always_inline)) {
        const int tok = c0 + (lane & (kChunk - 1));
        const int page = table[min(tok, t_end - 1) >> a.block_bits];
        const bool there = tok < t_end && page >= 0 && page < a.n_blocks;
        seen_next = (unsigned)__ballot(there);                       // (both halves of the wavefront hold the 32 tokens)
        slot_next = ((there ? page : 0) << a.block_bits) + (tok & in_page);   // (any page does for a token that is not counted)
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            // (a token that does not count takes its neighbour's codes: its pieces meet that token's in a matrix instruction, times zero)
            const int mine = wave * kOwn + i, from = seen_next >> mine & 1u ? mine : mine ^ 1;
            const int slot = __builtin_amdgcn_readlane(slot_next, from);
            const size_t rec = (((size_t)(slot >> a.block_bits) * a.Hkv + g) << a.block_bits) + (slot & in_page);
            const unsigned *k = reinterpret_cast<const unsigned *>(a.key_pages + rec * a.Mk) + gk, *v = reinterpret_cast<const unsigned *>(a.val_pages + rec * a.Mv) + gk;
            ck_next[i][0] = k[0];
            cv_next[i][0] = v[0];
            ck_next[i][1] = a.Mk == 32 ? k[4] : 0u;
            cv_next[i][1] = a.Mv == 32 ? v[4] : 0u;
        }
    };
    ask(t_begin);

    int t0[4] = {0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (a.turn && x < a.n_axes) t0[x] = a.node_pos[(size_t)s.n0 * a.n_axes + x];
    auto origin = [&](int ax) { return !AXES || ax == 0 ? t0[0] : ax == 1 ? t0[1] : ax == 2 ? t0[2] : t0[3]; };

    // queries, turned and scaled, as second operand: row n, elements 32 ks + 8 gk ..
    uint4_t qv[4], ql[4];
    const int r = r0 + wr * 16 + n;
    const int node = r / a.G, h = r % a.G;
    const bool there = r < R;
    const size_t at = (size_t)(s.n0 + (there ? node : 0)) * a.q_stride + (size_t)(g * a.G + h) * kD;
    const int32_t *pos = a.node_pos + (size_t)(s.n0 + (there ? node : 0)) * a.n_axes;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
        const uint4_t raw = *reinterpret_cast<const uint4_t *>(static_cast<const uint16_t *>(a.q) + at + 32 * ks + 8 * gk);
        uint4_t w, x;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = 16 * ks + 4 * gk + u, ax = AXES ? axis_of(a, j) : 0;
            float2 z = make_float2(bf16_lo(raw[u]), bf16_hi(raw[u]));
            if (a.turn) z = times(z, turned_by(a, pos[ax] - origin(ax), j));
            const uint2_t p = split_bf16(there ? z.x * a.scale2 : 0.f, there ? z.y * a.scale2 : 0.f);
            w[u] = p[0];
            x[u] = p[1];
        }
        qv[ks] = w;
        ql[ks] = x;
    }

    uint4_t sel;
    unsigned sidx;
    selection(lane, sel, sidx);
    const bf16x8_t selv = __builtin_bit_cast(bf16x8_t, sel);
    const int half = gk & 1, second = gk >> 1;      // the lane's 4 elements of a piece, and which token of a pair it ends up with
    const __amdgpu_buffer_rsrc_t krows = make_rsrc(static_cast<const uint16_t *>(a.key_cb) + (size_t)g * a.Mk * kK * kD, (unsigned)(a.Mk * kK * kD * 2));
    const __amdgpu_buffer_rsrc_t vrows = make_rsrc(static_cast<const uint16_t *>(a.val_cb) + (size_t)g * a.Mv * kK * kD, (unsigned)(a.Mv * kK * kD * 2));
    const unsigned lane_at = (unsigned)(4 * gk) * (kK * kD * 2) + (unsigned)n * 16u;

    floatx4_t o[NX];                                 // element 16 (wd NX + x) + 4 gk + i of row n
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < NX; ++x) o[x] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    // the sums of two tokens, by 16 codebooks
    auto fetch = [&](const __amdgpu_buffer_rsrc_t rows, unsigned code, int blk, uint4_t (&v)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 4; ++st)
            v[st] = __builtin_amdgcn_raw_buffer_load_b128(rows, lane_at + ((code >> (8 * st) & 255u) << 8), (16 * blk + st) * (kK * kD * 2), 0);
    };
    auto add = [&](floatx4_t acc, const uint4_t (&va)[4], const uint4_t (&vb)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            const uint8v_t both = {va[st][0], va[st][1], va[st][2], va[st][3], vb[st][0], vb[st][1], vb[st][2], vb[st][3]};
            acc = __builtin_amdgcn_smfmac_f32_16x16x64_bf16(selv, __builtin_bit_cast(bf16x16_t, both), acc, (int)sidx, 0, 0);
        }
        return acc;
    };
    auto decode = [&](const __amdgpu_buffer_rsrc_t rows, const unsigned (&c)[kOwn][2], int M, floatx4_t (&acc)[kOwn / 2]) __attribute__((always_inline)) {
        uint4_t v[kOwn][4];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) fetch(rows, c[i][0], 0, v[i]);
#pragma unroll
        for (int p = 0; p < kOwn / 2; ++p) acc[p] = add(floatx4_t{0.f, 0.f, 0.f, 0.f}, v[2 * p], v[2 * p + 1]);
        if (M == 32) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) fetch(rows, c[i][1], 1, v[i]);
#pragma unroll
            for (int p = 0; p < kOwn / 2; ++p) acc[p] = add(acc[p], v[2 * p], v[2 * p + 1]);
        }
    };

    for (int c0 = t_begin; c0 < t_end; c0 += kChunk) {
        unsigned ck[kOwn][2], cv[kOwn][2];
        const unsigned seen = seen_next;
        const int slot = slot_next;
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) { ck[i][k] = ck_next[i][k]; cv[i][k] = cv_next[i][k]; }
        if (c0 + kChunk < t_end) ask(c0 + kChunk);
        float2 e[kOwn / 2][2];
#pragma unroll
        for (int p = 0; p < kOwn / 2; ++p)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                e[p][u] = make_float2(1.f, 0.f);
                if (!a.turn) continue;
                const int mine = wave * kOwn + 2 * p + second, j = 4 * n + 2 * half + u, ax = AXES ? axis_of(a, j) : 0;
                int pos = c0 + mine;
                if (a.key_pos) pos = a.key_pos[(size_t)__shfl(slot, mine) * a.n_axes + ax];
                e[p][u] = turned_by(a, pos - origin(ax), j);
            }
        floatx4_t acc[kOwn / 2];
        decode(krows, ck, a.Mk, acc);
#pragma unroll
        for (int p = 0; p < kOwn / 2; ++p) {
            const float2 z0 = times(make_float2(acc[p][0], acc[p][1]), e[p][0]), z1 = times(make_float2(acc[p][2], acc[p][3]), e[p][1]);
            const uint2_t x = split_bf16(z0.x, z0.y), y = split_bf16(z1.x, z1.y);
#pragma unroll
            for (int k = 0; k < 2; ++k) *reinterpret_cast<uint2_t *>(ktile[k] + (wave * kOwn + 2 * p + second) * kRowBytes + n * 16 + half * 8) = uint2_t{x[k], y[k]};
        }
        decode(vrows, cv, a.Mv, acc);
#pragma unroll
        for (int p = 0; p < kOwn / 2; ++p) {
            const int mine = wave * kOwn + 2 * p + second;
            const bool counts = seen >> mine & 1u;   // (a weight of zero does not hide an infinity)
            const uint2_t x = split_bf16(acc[p][0], acc[p][1]), y = split_bf16(acc[p][2], acc[p][3]);
#pragma unroll
            for (int k = 0; k < 2; ++k) *reinterpret_cast<uint2_t *>(vtile[k] + mine * kRowBytes + n * 16 + half * 8) = uint2_t{counts ? x[k] : 0u, counts ? y[k] : 0u};
        }
        __syncthreads();
        floatx4_t sc[2];
        sc[0] = sc[1] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint4_t kv = *reinterpret_cast<const uint4_t *>(ktile[0] + (16 * t + n) * kRowBytes + 64 * ks + 16 * gk);
                const uint4_t kl = *reinterpret_cast<const uint4_t *>(ktile[1] + (16 * t + n) * kRowBytes + 64 * ks + 16 * gk);
                sc[t] = product(kv, kl, qv[ks], ql[ks], sc[t]);
            }
        uint4_t pv, pl;
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sc[t][i] = seen >> (16 * t + 4 * gk + i) & 1u ? sc[t][i] : -INFINITY;
                top = fmaxf(top, sc[t][i]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m, top), base = now == -INFINITY ? 0.f : now;
        const float old = __builtin_amdgcn_exp2f(m - base);
        m = now;
        float sum = 0.f, w[8];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[4 * t + i] = __builtin_amdgcn_exp2f(sc[t][i] - base);
                sum += w[4 * t + i];
            }
        l = l * old + sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2_t x = split_bf16(w[2 * i], w[2 * i + 1]);
            pv[i] = x[0];
            pl[i] = x[1];
        }
#pragma unroll
        for (int x = 0; x < NX; ++x) o[x] *= old;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            uint4_t vv[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const char *at = vtile[k] + (4 * gk + n / 4) * kRowBytes + 32 * (wd * NX + x) + 8 * (n & 3);
                const uint2_t v0 = lds_read_columns(at), v1 = lds_read_columns(at + 16 * kRowBytes);
                vv[k] = uint4_t{v0[0], v0[1], v1[0], v1[1]};
            }
            o[x] = product(vv[0], vv[1], pv, pl, o[x]);
        }
        if (c0 + kChunk < t_end) __syncthreads();
    }
    float sum = l;
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (r >= R) return;
    const size_t row = ((size_t)(s.n0 + r / a.G) * a.Hq + g * a.G + r % a.G) * a.splits + split;
#pragma unroll
    for (int x = 0; x < NX; ++x) *reinterpret_cast<floatx4_t *>(a.part + row * kD + 16 * (wd * NX + x) + 4 * gk) = o[x];
    if (gk == 0 && wd == 0) a.stat[row] = make_float2(m, sum);
}

// ------------------------------------------------------------------ k_tree_rows_f32
// The same in fp32 throughout, for fp32 queries or codebooks: four wavefronts with 16 rows each, 16 tokens at a time.  A thread decodes 8
// elements of a token by vector additions, keys first (32 fp32 codebooks of keys fill an L2; four wavefronts more for the values at the same time:
// one head, 5 rows, 4096 tokens 24 -> 30.6 us); products by v_mfma_f32_16x16x4_f32, whose operands have one element a lane, so that
// a weight is an operand of the second product as it is.
constexpr int kWideThreads = 256;
template <bool Q16, bool CB16>
__global__ __launch_bounds__(kWideThreads) void k_tree_rows_f32(const TreeArgs a)
{
    __shared__ __align__(16) float ktile[kWideChunk * kWideRow], vtile[kWideChunk * kWideRow];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int id = blockIdx.x;
    const int g = id % a.Hkv;
    id /= a.Hkv;
    const int rt = id % a.row_tiles;
    id /= a.row_tiles;
    const int split = id % a.splits, b = id / a.splits;
    const Span s = span_of(a, b);
    const int R = s.n * a.G, r0 = rt * 64, t_begin = split * a.split_len, t_end = min(s.L, t_begin + a.split_len);
    if (r0 >= R || t_begin >= t_end) return;
    const int n = lane & 15, gk = lane >> 4;
    const int r = r0 + wave * 16 + n;
    const bool row_there = r < R;
    const int node = s.n0 + (row_there ? r / a.G : 0), h = r % a.G;

    // row n, element 4 x + gk
    float qv[32];
#pragma unroll
    for (int x = 0; x < 32; ++x) {
        const int e = 4 * x + gk, j = e >> 1, ax = axis_of(a, j);
        const size_t at = (size_t)node * a.q_stride + (size_t)(g * a.G + h) * kD + 2 * j;
        float2 z = make_float2(cb_elem<Q16>(a.q, at), cb_elem<Q16>(a.q, at + 1));
        if (a.turn) z = times(z, turned_by(a, a.node_pos[(size_t)node * a.n_axes + ax] - a.node_pos[(size_t)s.n0 * a.n_axes + ax], j));
        qv[x] = row_there ? (e & 1 ? z.y : z.x) * a.scale2 : 0.f;
    }
    floatx4_t o[8];                                  // element 16 x + 4 gk + i
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) o[x] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    const int32_t *table = a.tables + (size_t)b * a.max_blocks;
    const int dt = tid >> 4, de = (tid & 15) * 8;   // the token and elements that this thread decodes
    for (int c0 = t_begin; c0 < t_end; c0 += kWideChunk) {
        const int tok = c0 + (lane & 15);
        const int pg = tok < t_end ? table[tok >> a.block_bits] : -1;
        const unsigned seen = (unsigned)__ballot(pg >= 0 && pg < a.n_blocks) & 0xffffu;
        const bool counts = seen >> dt & 1u;
        const int page = counts ? table[(c0 + dt) >> a.block_bits] : 0, in_page = (c0 + dt) & ((1 << a.block_bits) - 1);
        const size_t rec = (((size_t)page * a.Hkv + g) << a.block_bits) + in_page;
        // (all codes of the record are asked for at once, rows eight books at a time)
        auto decode = [&](const uint8_t *codes, const void *cb, int M, float *acc) __attribute__((always_inline)) {
            uint4_t w[2];
            w[0] = *reinterpret_cast<const uint4_t *>(codes);
            w[1] = M == 32 ? *reinterpret_cast<const uint4_t *>(codes + 16) : w[0];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
                if (c >= M) break;
                __builtin_amdgcn_sched_barrier(0);
                uint4_t x[8][CB16 ? 1 : 2];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const unsigned code = w[c / 16][(c % 16 + u) / 4] >> (8 * (u & 3)) & 255u;
                    const size_t at = (((size_t)g * M + c + u) * kK + code) * kD + de;
                    if constexpr (CB16) {
                        x[u][0] = *reinterpret_cast<const uint4_t *>(static_cast<const uint16_t *>(cb) + at);
                    } else {
                        x[u][0] = *reinterpret_cast<const uint4_t *>(static_cast<const float *>(cb) + at);
                        x[u][1] = *reinterpret_cast<const uint4_t *>(static_cast<const float *>(cb) + at + 4);
                    }
                }
#pragma unroll
                for (int u = 0; u < 8; ++u)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if constexpr (CB16) {
                            const unsigned v = x[u][0][e / 2];
                            acc[e] += e & 1 ? bf16_hi(v) : bf16_lo(v);
                        } else {
                            const unsigned v = x[u][e / 4][e & 3];
                            acc[e] += __builtin_bit_cast(float, v);
                        }
                    }
            }
        };
        float x[8];
        decode(a.key_pages + rec * a.Mk, a.key_cb, a.Mk, x);
        if (a.turn) {
            const int32_t *own = a.key_pos ? a.key_pos + (((size_t)page << a.block_bits) + in_page) * a.n_axes : nullptr;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = de / 2 + u, ax = axis_of(a, j);
                const float2 z = times(make_float2(x[2 * u], x[2 * u + 1]), turned_by(a, (own ? own[ax] : c0 + dt) - a.node_pos[(size_t)s.n0 * a.n_axes + ax], j));
                x[2 * u] = z.x;
                x[2 * u + 1] = z.y;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ktile[dt * kWideRow + de + e] = x[e];
        decode(a.val_pages + rec * a.Mv, a.val_cb, a.Mv, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) vtile[dt * kWideRow + de + e] = counts ? x[e] : 0.f;   // (a weight of zero does not hide an infinity)
        __syncthreads();
        floatx4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 32; ++k) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(ktile[n * kWideRow + 4 * k + gk], qv[k], sc, 0, 0, 0);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!(seen >> (4 * gk + i) & 1u)) sc[i] = -INFINITY;
            top = fmaxf(top, sc[i]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m, top), base = now == -INFINITY ? 0.f : now, old = __builtin_amdgcn_exp2f(m - base);
        m = now;
        float w[4], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[i] = __builtin_amdgcn_exp2f(sc[i] - base); sum += w[i]; }
        l = l * old + sum;
#pragma unroll
        for (int y = 0; y < 8; ++y) {
            o[y] *= old;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[y] = __builtin_amdgcn_mfma_f32_16x16x4f32(vtile[(4 * gk + i) * kWideRow + 16 * y + n], w[i], o[y], 0, 0, 0);
        }
        __syncthreads();
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (!row_there) return;
    const size_t row = ((size_t)node * a.Hq + g * a.G + h) * a.splits + split;
#pragma unroll
    for (int y = 0; y < 8; ++y) *reinterpret_cast<floatx4_t *>(a.part + row * kD + 16 * y + 4 * gk) = o[y];
    if (gk == 0) a.stat[row] = make_float2(m, l);
}

}  // namespace

#include "commvq_tree_dense.hpp"
#include "commvq_tree_stream.hpp"

namespace {

// ------------------------------------------------------------------ k_tree_final
// A workgroup joins the parts of one row: a wavefront a run of ranges and every W-th node that the row attends to, a lane one sub-space.
// The nodes' part is fp32 arithmetic, node by node: nodes outside the mask are not read, so that what they hold cannot matter.
// Bound by latency: the ranges' statistics are one load of the wavefront, their rows are asked for eight at a time, nodes two at a time.  Measured: 256 rows
// of 8 nodes and 22 ranges 5.3 us, 832 of 26 and 32 9.3, 2048 of 64 and 32 12.4.
template <bool Q16, int W>
__global__ __launch_bounds__(64 * W) void k_tree_final(const TreeArgs a)
{
    __shared__ float sm[W], sl[W];
    __shared__ float2 so[W][kJ];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int node = blockIdx.x / a.Hq, h = blockIdx.x % a.Hq, g = h / a.G;
    // the sequence: as many as end at or before this node come before it
    int b = 0;
    for (int c = 0; c < a.batch; c += 64) {
        const int x = c + lane;
        const int ended = __popcll(__ballot(x < a.batch && a.cu[x + 1] <= node));
        b += ended;
        if (ended < 64) break;
    }
    if (b >= a.batch) return;                         // a row behind the last sequence
    const Span s = span_of(a, b);
    const int i = node - s.n0;
    const bool there = i >= 0 && i < s.n;
    float m = -INFINITY, l = 0.f;
    float2 o = make_float2(0.f, 0.f);

    // nodes
    unsigned long long mask = !there ? 0 : a.mask ? a.mask[node] : ~0ull >> (63 - i);
    if (s.n < 64) mask &= (1ull << s.n) - 1;
    const int ax = axis_of(a, lane);
    const size_t at = (size_t)node * a.q_stride + (size_t)h * kD + 2 * lane;
    const float2 q = make_float2(cb_elem<Q16>(a.q, at) * a.scale2, cb_elem<Q16>(a.q, at + 1) * a.scale2);
    const int own = a.turn ? a.node_pos[(size_t)node * a.n_axes + ax] : 0;
    for (int k = 0; k < wave; ++k) mask &= mask - 1;  // (a wavefront's first node)
    while (mask) {
        constexpr int U = 2;
        float2 key[U], val[U], e[U];
        bool is[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            is[u] = mask != 0;
            const int j = s.n0 + (is[u] ? __builtin_ctzll(mask) : 0);
            const size_t from = (size_t)j * a.node_stride + (size_t)g * kD + 2 * lane;
            key[u] = make_float2(cb_elem<Q16>(a.node_k, from), cb_elem<Q16>(a.node_k, from + 1));
            val[u] = make_float2(cb_elem<Q16>(a.node_v, from), cb_elem<Q16>(a.node_v, from + 1));
            e[u] = a.turn ? turned_by(a, own - a.node_pos[(size_t)j * a.n_axes + ax], lane) : make_float2(1.f, 0.f);
#pragma unroll
            for (int k = 0; k < W; ++k) mask &= mask - 1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!is[u]) break;
            const float2 z = times(q, e[u]);
            const float x = wave_sum(z.x * key[u].x + z.y * key[u].y);
            const float now = fmaxf(m, x), base = now == -INFINITY ? 0.f : now;
            const float was = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(x - base);
            m = now;
            l = l * was + w;
            o.x = o.x * was + val[u].x * w;
            o.y = o.y * was + val[u].y * w;
        }
    }

    // ranges: those of a wavefront follow each other, 64 at a time
    const int ns = there ? min((s.L + a.split_len - 1) / a.split_len * a.halves, a.splits) : 0, per = (ns + W - 1) / W;
    const size_t row = (size_t)blockIdx.x * a.splits;
    const int k_end = min(ns, (wave + 1) * per);
    for (int k0 = wave * per; k0 < k_end; k0 += 64) {
        const int here = min(64, k_end - k0);
        const float2 st = lane < here ? a.stat[row + k0 + lane] : make_float2(-INFINITY, 0.f);
        const float now = fmaxf(m, wave_max(st.x)), base = now == -INFINITY ? 0.f : now;
        const float was = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(st.x - base);   // (a range without a page: 0)
        m = now;
        l = l * was + wave_sum(st.y * w);
        o.x *= was;
        o.y *= was;
        const float *from = a.part + (row + k0) * kD + 2 * lane;
        for (int k = 0; k < here; k += 8) {
            float2 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const float2 *>(from + (size_t)min(k + u, here - 1) * kD);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), min(k + u, here - 1)));
                if (k + u >= here) break;
                o.x += v[u].x * f;
                o.y += v[u].y * f;
            }
        }
    }
    if (lane == 0) { sm[wave] = m; sl[wave] = l; }
    so[wave][lane] = o;
    __syncthreads();
    if (wave) return;
    float top = -INFINITY, sum = 0.f;
    float2 t = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, sm[w]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        if (sl[w] == 0.f) continue;                   // (nothing there)
        const float f = __builtin_amdgcn_exp2f(sm[w] - top);
        sum += sl[w] * f;
        t.x += so[w][lane].x * f;
        t.y += so[w][lane].y * f;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that attends to nothing: zeros
    if (Q16) static_cast<unsigned *>(a.out)[(size_t)blockIdx.x * kJ + lane] = pack_bf16(t.x * inv, t.y * inv);
    else static_cast<float2 *>(a.out)[(size_t)blockIdx.x * kJ + lane] = make_float2(t.x * inv, t.y * inv);
}

// ------------------------------------------------------------------ k_tree_pack
// A codebook in the order in which it is streamed through LDS: packed[head][slice][block of 16 books][word][16 books], pieces of 16 bytes,
// slice = 8 consecutive elements of every codeword.  One thread per piece of the source.
__global__ __launch_bounds__(256) void k_tree_pack(const uint4 *__restrict__ cb, uint4 *__restrict__ packed, int M, size_t pieces)
{
    const size_t t = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= pieces) return;
    const int sl = (int)(t & 15);
    const size_t row = t >> 4;                  // (head * M + book) * 256 + word
    const int word = (int)(row & (kK - 1));
    const size_t hm = row / kK;
    const int m = (int)(hm % M);
    const size_t g = hm / M;
    packed[(((g * 16 + sl) * (M / 16) + m / 16) * kK + word) * 16 + m % 16] = cb[t];
}

// The power of two that brings sums of M codewords of a head to at most 2^14, so that turned keys (sqrt 2 more) and values fit fp16 whatever the codes
// and keep its 11 bits down to 2^-28 of that.  A workgroup per (head, codebook kind); numbers that are not finite do not count.
__global__ __launch_bounds__(1024) void k_tree_scale(const uint4 *__restrict__ cb, float *__restrict__ scales, int M)
{
    __shared__ float waves[16];
    const int n = M * kK * kD / 8;
    const uint4 *from = cb + (size_t)blockIdx.x * n;
    float top = 0.f;
    for (int i = threadIdx.x; i < n; i += 1024) {
        const uint4 v = from[i];
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = fabsf(bf16_lo(w[k])), b = fabsf(bf16_hi(w[k]));
            top = fmaxf(top, a < INFINITY ? a : 0.f);
            top = fmaxf(top, b < INFINITY ? b : 0.f);
        }
    }
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 16; ++w) top = fmaxf(top, waves[w]);
    int e = 0;
    if (top > 0.f) (void)frexpf(top, &e);            // top < 2^e
    int m = 0;
    while (1 << m < M) ++m;
    scales[2 * blockIdx.x] = ldexpf(1.f, min(max(14 - e - m, -100), 100));
}

// ------------------------------------------------------------------ host side
struct TreePlan {
    int nr;              // rows gathered: row tiles of a workgroup; streamed: sets of a tile; decoded ahead: wavefronts of different rows
    int sets;            // decoded ahead: sets of a tile
    int row_tiles, splits, split_len;
    int tiles_per_head;  // decoded ahead: row tiles of 16 of all sequences
    int pass_tiles, passes;  // decoded ahead: token tiles of a pass
    size_t stat_at, q_at, q_scales_at, keys_at, vals_at, seen_at, phases_at, bytes;
};

inline size_t tree_packed_bytes(const commvq_config &c) { return (size_t)c.n_kv_heads * (c.m_key + c.m_val) * kK * kD * 2; }
inline bool wide(const commvq_config &c) { return c.q_dtype != COMMVQ_BF16 || c.codebook_dtype != COMMVQ_BF16; }

void tree_room(const commvq_handle *h, int batch, int total_nodes, bool stream, TreePlan &p)
{
    const size_t parts = (size_t)total_nodes * h->cfg.n_q_heads * p.splits;
    p.stat_at = align_up(parts * kD * 4, 256);
    p.q_at = align_up(p.stat_at + parts * 8, 256);
    p.tiles_per_head = first_tile(total_nodes, h->G, batch) + 1;
    p.bytes = std::max<size_t>(256, stream ? p.q_at + (size_t)p.tiles_per_head * h->cfg.n_kv_heads * 4096 : p.q_at);
}

// Rows of a workgroup: the smallest of 16, 32, 64 and 128 that holds the largest tree's, or 128.  Ranges: in whole chunks, as many as give
// every compute unit four workgroups.
TreePlan rows_plan(const commvq_handle *h, int batch, int total_nodes, int max_nodes, int max_seqlen)
{
    TreePlan p{};
    const int rows = max_nodes * h->G;
    p.nr = rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
    if (wide(h->cfg)) p.nr = 4;
    p.row_tiles = (rows + 16 * p.nr - 1) / (16 * p.nr);
    const int chunk = wide(h->cfg) ? kWideChunk : kChunk;
    const int64_t units = (int64_t)batch * h->cfg.n_kv_heads * p.row_tiles;
    const int64_t chunks = (max_seqlen + chunk - 1) / chunk;
    const int64_t want = std::max<int64_t>(1, 1024 / units);
    const int64_t per = std::max<int64_t>(1, (chunks + want - 1) / want);
    p.split_len = (int)per * chunk;
    p.splits = (int)((chunks + per - 1) / per);
    tree_room(h, batch, total_nodes, false, p);
    return p;
}

// Tiles and ranges of k_tree_stream: of the tile sizes the one, and of whole tiles so many a workgroup, that the last round of workgroups (one
// per compute unit) ends soonest, of the sixteen lowest numbers of rounds.  A stage of 512, 1024 and 2048 tokens takes 0.9, 1.2 and 2.0 us (the first two wait for the transfer of the
// next one): 16 codebooks each, 8 heads, whole calls with tiles of 512 | 1024 | 2048: 16 000 tokens 42.5 | 45.8 | 70.0 us, 32 768 77.9 | 51.4 | 73.2,
// 65 536 146 | 99.1 | 83.5.
TreePlan stream_plan(const commvq_handle *h, int batch, int total_nodes, int max_seqlen)
{
    TreePlan p{};
    p.row_tiles = 1;
    const int64_t units = (int64_t)batch * h->cfg.n_kv_heads;
    double best = 0;
    for (int sets = kStreamMaxSets; sets >= 2; sets /= 2) {
        const int64_t tiles = (max_seqlen + stream_tile(sets) - 1) / stream_tile(sets);
        const double tile_us = (h->cfg.m_key + h->cfg.m_val) * (sets == 8 ? 2.0 : sets == 4 ? 1.2 : 0.9);
        for (int64_t rounds = (units + 255) / 256, last = rounds + 16; rounds < last; ++rounds) {
            const int64_t most = std::min(256 * rounds / units, tiles), x = (tiles + most - 1) / most;   // ranges of a sequence, tiles of a range
            const double cost = (double)((units * ((tiles + x - 1) / x) + 255) / 256) * (x * tile_us + 3.0);
            if (p.nr == 0 || cost < best) {
                best = cost;
                p.nr = sets;
                p.split_len = (int)x * stream_tile(sets);
                p.splits = (int)((tiles + x - 1) / x);
            }
        }
    }
    tree_room(h, batch, total_nodes, false, p);
    return p;
}

// Decoded ahead: passes over as many tiles as the scratch holds, which is 128 (tile, head)s, 128 MiB: what the 256 MiB behind the L2s hold from
// one kernel to the next (decoding 128K tokens of 8 heads: 161 us in four such passes, 252 in two of twice the size, 217 in one).
constexpr int kDenseTileHeads = 128;
TreePlan dense_plan(const commvq_handle *h, int batch, int total_nodes, int max_nodes, int max_seqlen)
{
    TreePlan p{};
    const int rows = max_nodes * h->G, groups = (rows + 16 * kDenseRows - 1) / (16 * kDenseRows), Hkv = h->cfg.n_kv_heads;
    p.nr = groups <= 1 ? 1 : groups <= 2 ? 2 : groups <= 4 ? 4 : 8;
    p.row_tiles = (groups + p.nr - 1) / p.nr;
    // tiles of 1024 tokens instead of 2048 where that saves rounds of workgroups: 0.62 of a large one's time (8 heads, 8 nodes, 16 codebooks, 1024 | 2048:
    // 8000 tokens 53.8 | 59.3 us, 32 768 104.9 | 85.4; 32 sequences of 600 118.6 | 173.0, of 1500 204.6 | 174.3)
    auto rounds = [&](int sets) { return ((int64_t)batch * ((max_seqlen + sets * kDecodeSetTokens - 1) / (sets * kDecodeSetTokens)) * Hkv * 2 + 255) / 256; };
    p.sets = 0.62 * (double)rounds(2) < (double)rounds(4) ? 2 : 4;
    const int tile = p.sets * kDecodeSetTokens, halves = p.sets * kDecodeWaves / kDenseSteps, tiles = (max_seqlen + tile - 1) / tile;
    const int64_t all = (int64_t)batch * tiles;
    p.pass_tiles = (int)std::min<int64_t>(all, std::max(1, kDenseTileHeads * kDecodeMaxSets / p.sets / Hkv));
    p.passes = (int)((all + p.pass_tiles - 1) / p.pass_tiles);
    p.split_len = tile;
    p.splits = std::min(tiles, p.pass_tiles) * halves;
    tree_room(h, batch, total_nodes, true, p);
    const size_t steps = (size_t)p.pass_tiles * Hkv * p.sets * kDecodeWaves;
    p.q_scales_at = align_up(p.bytes, 256);
    p.keys_at = align_up(p.q_scales_at + (size_t)p.tiles_per_head * Hkv * 64, 256);
    p.vals_at = p.keys_at + steps * kStepBytes;
    p.seen_at = p.vals_at + steps * kStepBytes;
    p.phases_at = align_up(p.seen_at + steps * 4, 256);
    p.bytes = p.phases_at + (size_t)p.pass_tiles * p.sets * kDecodeWaves * 16 * 64 * 16;
    return p;
}

// Which kernels a call takes.  (What the workspace is sized for does not depend on tables and positions, which are not known then.)  With u tokens
// times KV heads, M the mean number of codebooks, 8 heads, rows gathered | the other way: up to 16 rows, M = 16: u = 16 000 28.6 | 36.4 us, 32 000
// 48.5 | 37.1; M = 32: 32 000 62.7 | 73.1, 64 000 90.6 | 74.5.  32 rows, M = 16: 16 000 32.2 | 49.0, 32 000 54.7 | 50.9; 256 rows 66.5 | 86.4, 120 | 90.1;
// M = 32: 72.2 | 104, 134 | 106.
enum Way { kRows, kStream, kDense };
Way tree_way(const commvq_handle *h, int batch, int max_nodes, int max_seqlen, bool tables, bool implicit)
{
    if (wide(h->cfg) || !tables || max_seqlen < 1) return kRows;
    const int64_t units = (int64_t)batch * h->cfg.n_kv_heads * max_seqlen;
    if (max_nodes * h->G <= kStreamRows && implicit) return units < 650 * (h->cfg.m_key + h->cfg.m_val) ? kRows : kStream;
    return units < 26000 ? kRows : kDense;
}

TreePlan plan_of(Way way, const commvq_handle *h, int batch, int total_nodes, int max_nodes, int max_seqlen)
{
    return way == kStream ? stream_plan(h, batch, total_nodes, max_seqlen) : way == kDense ? dense_plan(h, batch, total_nodes, max_nodes, max_seqlen)
                                                                           : rows_plan(h, batch, total_nodes, max_nodes, max_seqlen);
}

commvq_status check_tree_sizes(const commvq_handle *h, int32_t batch, int32_t total_nodes, int32_t max_nodes, int32_t max_seqlen)
{
    if (h->cfg.key_format != COMMVQ_KEYS_INDEXED || h->cfg.value_format != COMMVQ_VALUES_INDEXED) return COMMVQ_ERR_CONFIG;
    if (batch < 1 || max_nodes < 1 || max_nodes > kMaxNodes || total_nodes < max_nodes || (int64_t)total_nodes > (int64_t)batch * max_nodes) return COMMVQ_ERR_SHAPE;
    if (max_seqlen < 0 || max_seqlen > 1 << 30) return COMMVQ_ERR_SHAPE;
    if ((int64_t)total_nodes * h->cfg.n_q_heads > 0x7fffffff) return COMMVQ_ERR_SHAPE;  // workgroups of the last kernel
    return COMMVQ_OK;
}

template <int NR>
hipError_t launch_rows(const TreeArgs &a, dim3 grid, hipStream_t s)
{
    if (a.n_axes > 1) k_tree_rows<NR, true><<<grid, 64 * kRowsWaves, 0, s>>>(a);
    else k_tree_rows<NR, false><<<grid, 64 * kRowsWaves, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_wide(const TreeArgs &a, dim3 grid, hipStream_t s)
{
    if (a.q_bf16) k_tree_rows_f32<true, false><<<grid, kWideThreads, 0, s>>>(a);
    else if (a.cb_bf16) k_tree_rows_f32<false, true><<<grid, kWideThreads, 0, s>>>(a);
    else k_tree_rows_f32<false, false><<<grid, kWideThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <int NBK, int NBV, int SETS>
hipError_t launch_stream_as(const TreeArgs &a, const char *tables, dim3 grid, hipStream_t s)
{
    static std::atomic<uint64_t> lds_ok{0};
    const hipError_t e = allow_dynamic_lds(k_tree_stream<NBK, NBV, SETS>, kTreeLds, lds_ok);
    if (e != hipSuccess) return e;
    k_tree_stream<NBK, NBV, SETS><<<grid, kStreamThreads, kTreeLds, s>>>(a, tables);
    return hipGetLastError();
}

template <int NBK, int NBV>
hipError_t launch_stream_sets(const TreeArgs &a, int sets, const char *tables, dim3 grid, hipStream_t s)
{
    return sets == 8 ? launch_stream_as<NBK, NBV, 8>(a, tables, grid, s) : sets == 4 ? launch_stream_as<NBK, NBV, 4>(a, tables, grid, s)
                                                                          : launch_stream_as<NBK, NBV, 2>(a, tables, grid, s);
}

hipError_t launch_stream(const TreeArgs &a, int sets, const char *tables, dim3 grid, hipStream_t s)
{
    if (a.Mk == 16) return a.Mv == 16 ? launch_stream_sets<1, 1>(a, sets, tables, grid, s) : launch_stream_sets<1, 2>(a, sets, tables, grid, s);
    return a.Mv == 16 ? launch_stream_sets<2, 1>(a, sets, tables, grid, s) : launch_stream_sets<2, 2>(a, sets, tables, grid, s);
}

bool explicit_positions(const TreeArgs &a) { return a.turn && (a.key_pos || a.n_axes > 1); }

template <int NBK, int NBV, int SETS, bool EXPLICIT>
hipError_t launch_decode_as(const TreeArgs &a, const DensePass &d, const char *tables, dim3 grid, hipStream_t s)
{
    static std::atomic<uint64_t> lds_ok{0};
    const hipError_t e = allow_dynamic_lds(k_tree_decode<NBK, NBV, SETS, EXPLICIT>, kDecodeLds, lds_ok);
    if (e != hipSuccess) return e;
    k_tree_decode<NBK, NBV, SETS, EXPLICIT><<<grid, kDecodeThreads, kDecodeLds, s>>>(a, d, tables);
    return hipGetLastError();
}

template <int NBK, int NBV>
hipError_t launch_decode(const TreeArgs &a, const DensePass &d, const char *tables, dim3 grid, hipStream_t s)
{
    if (explicit_positions(a)) return d.sets == 4 ? launch_decode_as<NBK, NBV, 4, true>(a, d, tables, grid, s) : launch_decode_as<NBK, NBV, 2, true>(a, d, tables, grid, s);
    return d.sets == 4 ? launch_decode_as<NBK, NBV, 4, false>(a, d, tables, grid, s) : launch_decode_as<NBK, NBV, 2, false>(a, d, tables, grid, s);
}

template <int WR>
hipError_t launch_dense_as(const TreeArgs &a, const DensePass &d, dim3 grid, hipStream_t s)
{
    static std::atomic<uint64_t> lds_ok{0};
    const hipError_t e = allow_dynamic_lds(k_tree_dense<WR>, dense_lds(WR), lds_ok);
    if (e != hipSuccess) return e;
    k_tree_dense<WR><<<grid, 64 * kDenseWaves, dense_lds(WR), s>>>(a, d);
    return hipGetLastError();
}

hipError_t launch_dense(const TreeArgs &a, const TreePlan &p, int passes, const char *tables, char *workspace, hipStream_t s)
{
    DensePass d{workspace + p.keys_at, workspace + p.vals_at, reinterpret_cast<unsigned *>(workspace + p.seen_at),
                reinterpret_cast<floatx4_t *>(workspace + p.phases_at), reinterpret_cast<uint4_t *>(workspace + p.q_at), reinterpret_cast<float *>(workspace + p.q_scales_at),
                p.tiles_per_head, 0, p.pass_tiles, p.sets, p.sets * kDecodeSetTokens, p.sets * kDecodeWaves, 0, (a.max_nodes * a.G + 15) / 16};
    const int64_t turns = ((int64_t)a.batch * a.Hkv * d.turn_tiles + kDecodeWaves - 1) / kDecodeWaves;
    const int64_t decode = 2ll * d.tiles * a.Hkv, dense = (int64_t)d.tiles * a.Hkv * p.row_tiles * (d.steps / kDenseSteps);
    if (std::max(turns + decode, dense) > 0x7fffffff) return hipErrorInvalidValue;
    for (int i = 0; i < passes; ++i, d.tile0 += d.tiles) {
        d.turn_wgs = i == 0 ? (int)turns : 0;
        const dim3 first((unsigned)(d.turn_wgs + decode)), second((unsigned)dense);
        hipError_t e;
        if (explicit_positions(a)) {
            k_tree_phases<<<dim3((unsigned)(d.tiles * d.steps)), 256, 0, s>>>(a, d);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (a.Mk == 16) e = a.Mv == 16 ? launch_decode<1, 1>(a, d, tables, first, s) : launch_decode<1, 2>(a, d, tables, first, s);
        else e = a.Mv == 16 ? launch_decode<2, 1>(a, d, tables, first, s) : launch_decode<2, 2>(a, d, tables, first, s);
        if (e != hipSuccess) return e;
        e = p.nr == 1 ? launch_dense_as<1>(a, d, second, s) : p.nr == 2 ? launch_dense_as<2>(a, d, second, s) : p.nr == 4 ? launch_dense_as<4>(a, d, second, s)
                                                                                                          : launch_dense_as<8>(a, d, second, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

bool misaligned(std::initializer_list<const void *> ps)
{
    uintptr_t all = 0;
    for (const void *p : ps) all |= reinterpret_cast<uintptr_t>(p);
    return (all & 15u) != 0;
}

}  // namespace

extern "C" {

commvq_status commvq_tree_workspace_bytes(const commvq_handle *h, int32_t batch, int32_t total_nodes, int32_t max_nodes,
                                          int32_t max_seqlen, size_t *bytes)
{
    if (!h || !bytes) return COMMVQ_ERR_NULL;
    const commvq_status st = check_tree_sizes(h, batch, total_nodes, max_nodes, max_seqlen);
    if (st != COMMVQ_OK) return st;
    *bytes = 0;
    for (const bool tables : {false, true})
        for (const bool implicit : {false, true})
            *bytes = std::max(*bytes, plan_of(tree_way(h, batch, max_nodes, max_seqlen, tables, implicit), h, batch, total_nodes, max_nodes, max_seqlen).bytes);
    return COMMVQ_OK;
}

commvq_status commvq_tree_attn(commvq_handle *h, const commvq_pages *pages, const commvq_tree *t, const void *q,
                               const void *node_keys, const void *node_vals, const uint8_t *key_pages,
                               const uint8_t *val_pages, const void *key_cb, const void *val_cb, const void *tables,
                               void *out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!h || !t || !q || !node_keys || !node_vals || !key_pages || !val_pages || !key_cb || !val_cb || !out) return COMMVQ_ERR_NULL;
    if (!t->seq_lens || !t->block_tables || !t->cu_nodes || !t->node_pos) return COMMVQ_ERR_NULL;
    commvq_status st = commvq_check_pages(pages);
    if (st != COMMVQ_OK) return st;
    if (pages->n_axes > 1 && !t->pair_axis) return COMMVQ_ERR_NULL;
    st = check_tree_sizes(h, t->batch, t->total_nodes, t->max_nodes, t->max_seqlen);
    if (st != COMMVQ_OK) return st;
    const commvq_config &c = h->cfg;
    if (tables && c.codebook_dtype != COMMVQ_BF16) return COMMVQ_ERR_CONFIG;
    if ((int64_t)t->max_seqlen > (int64_t)pages->max_blocks * pages->block_size) return COMMVQ_ERR_SHAPE;
    // keys at positions 0 .. L - 1 and nodes at or after the last of them
    if (!t->key_pos && !c.position_free && (int64_t)t->max_seqlen - 1 > c.max_position) return COMMVQ_ERR_SHAPE;
    if (t->total_tokens && (t->total_tokens < t->max_seqlen || t->total_tokens > (int64_t)t->batch * t->max_seqlen)) return COMMVQ_ERR_SHAPE;
    if (misaligned({q, node_keys, node_vals, key_pages, val_pages, key_cb, val_cb, tables, out})) return COMMVQ_ERR_SHAPE;
    const int64_t q_row = (int64_t)c.n_q_heads * kD, node_row = (int64_t)c.n_kv_heads * kD;
    if (t->q_stride && (t->q_stride < q_row || t->q_stride % 8)) return COMMVQ_ERR_SHAPE;
    if (t->node_stride && (t->node_stride < node_row || t->node_stride % 8)) return COMMVQ_ERR_SHAPE;
    TreeArgs a{};
    if (t->pair_axis)
        for (int j = 0; j < kJ; ++j) {
            if (t->pair_axis[j] >= pages->n_axes) return COMMVQ_ERR_SHAPE;
            a.axes[j >> 4] |= (unsigned)t->pair_axis[j] << (2 * (j & 15));
        }
    size_t need = 0;
    st = commvq_tree_workspace_bytes(h, t->batch, t->total_nodes, t->max_nodes, t->max_seqlen, &need);
    if (st != COMMVQ_OK) return st;
    const Way way = tree_way(h, t->batch, t->max_nodes, t->max_seqlen, tables != nullptr, pages->n_axes == 1 && !t->key_pos);
    const TreePlan p = plan_of(way, h, t->batch, t->total_nodes, t->max_nodes, t->max_seqlen);
    // (what the device may hold of it beyond this is left out: whole tiles, sequence by sequence)
    const int64_t tiles = t->total_tokens ? std::min<int64_t>((int64_t)p.pass_tiles * p.passes, t->total_tokens / std::max(1, p.split_len) + t->batch) : (int64_t)p.pass_tiles * p.passes;
    const int64_t wgs = (int64_t)t->batch * c.n_kv_heads * p.row_tiles * p.splits;
    if (wgs > 0x7fffffff) return COMMVQ_ERR_SHAPE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < need) return COMMVQ_ERR_WORKSPACE;
    if (h->device < 0) return COMMVQ_ERR_NO_DEVICE;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != h->device) return COMMVQ_ERR_NO_DEVICE;  // the phase tables are another GPU's
    a.q = q; a.node_k = node_keys; a.node_v = node_vals; a.key_pages = key_pages; a.val_pages = val_pages; a.key_cb = key_cb; a.val_cb = val_cb;
    a.seq_lens = t->seq_lens; a.tables = t->block_tables; a.cu = t->cu_nodes; a.node_pos = t->node_pos; a.key_pos = t->key_pos;
    a.mask = reinterpret_cast<const unsigned long long *>(t->node_mask);
    if (tables) a.scales = reinterpret_cast<const float *>(static_cast<const char *>(tables) + tree_packed_bytes(c));
    a.tbl_hi = h->tbl_hi; a.tbl_lo = h->tbl_lo;
    a.part = static_cast<float *>(workspace);
    a.stat = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + p.stat_at);
    a.out = out;
    a.q_stride = t->q_stride ? t->q_stride : q_row; a.node_stride = t->node_stride ? t->node_stride : node_row;
    a.batch = t->batch; a.Hq = c.n_q_heads; a.Hkv = c.n_kv_heads; a.G = h->G; a.Mk = c.m_key; a.Mv = c.m_val; a.n_hi = h->n_hi;
    a.n_axes = pages->n_axes; a.block_bits = __builtin_ctz((unsigned)pages->block_size); a.n_blocks = pages->n_blocks; a.max_blocks = pages->max_blocks;
    a.total_nodes = t->total_nodes; a.max_nodes = t->max_nodes; a.max_seqlen = t->max_seqlen;
    a.splits = p.splits; a.split_len = p.split_len; a.row_tiles = p.row_tiles; a.halves = way == kDense ? p.sets * kDecodeWaves / kDenseSteps : 1;
    a.turn = !c.position_free; a.q_bf16 = c.q_dtype == COMMVQ_BF16; a.cb_bf16 = c.codebook_dtype == COMMVQ_BF16;
    a.scale2 = h->scale * kLog2e;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (wgs > 0) {
        const dim3 grid((unsigned)wgs);
        hipError_t e;
        if (way == kDense) e = launch_dense(a, p, (int)((tiles + p.pass_tiles - 1) / p.pass_tiles), static_cast<const char *>(tables), static_cast<char *>(workspace), s);
        else if (way == kStream) e = launch_stream(a, p.nr, static_cast<const char *>(tables), grid, s);
        else if (wide(c)) e = launch_wide(a, grid, s);
        else if (p.nr == 1) e = launch_rows<1>(a, grid, s);
        else if (p.nr == 2) e = launch_rows<2>(a, grid, s);
        else if (p.nr == 4) e = launch_rows<4>(a, grid, s);
        else e = launch_rows<8>(a, grid, s);
        if (e != hipSuccess) return COMMVQ_ERR_LAUNCH;
    }
    const dim3 rows((unsigned)((int64_t)t->total_nodes * c.n_q_heads));
    // sixteen wavefronts a row where there are many ranges or few rows
    const bool many = p.splits > 32 && (int64_t)t->total_nodes * c.n_q_heads <= 1024;
    if (many) {
        if (a.q_bf16) k_tree_final<true, 16><<<rows, 64 * 16, 0, s>>>(a);
        else k_tree_final<false, 16><<<rows, 64 * 16, 0, s>>>(a);
    } else {
        if (a.q_bf16) k_tree_final<true, 4><<<rows, 64 * 4, 0, s>>>(a);
        else k_tree_final<false, 4><<<rows, 64 * 4, 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? COMMVQ_OK : COMMVQ_ERR_LAUNCH;
}

commvq_status commvq_tree_table_bytes(const commvq_handle *h, size_t *bytes)
{
    if (!h || !bytes) return COMMVQ_ERR_NULL;
    const commvq_config &c = h->cfg;
    if (c.codebook_dtype != COMMVQ_BF16 || c.key_format != COMMVQ_KEYS_INDEXED || c.value_format != COMMVQ_VALUES_INDEXED) return COMMVQ_ERR_CONFIG;
    *bytes = tree_packed_bytes(c) + align_up((size_t)c.n_kv_heads * 8, 256);
    return COMMVQ_OK;
}

commvq_status commvq_tree_prepare(commvq_handle *h, const void *key_cb, const void *val_cb, void *tables, void *stream)
{
    if (!h || !key_cb || !val_cb || !tables) return COMMVQ_ERR_NULL;
    size_t bytes = 0;
    const commvq_status st = commvq_tree_table_bytes(h, &bytes);
    if (st != COMMVQ_OK) return st;
    if (misaligned({key_cb, val_cb, tables})) return COMMVQ_ERR_SHAPE;
    if (h->device < 0) return COMMVQ_ERR_NO_DEVICE;
    const commvq_config &c = h->cfg;
    const size_t kp = (size_t)c.n_kv_heads * c.m_key * kK * 16, vp = (size_t)c.n_kv_heads * c.m_val * kK * 16;
    if (std::max(kp, vp) / 256 > 0x7fffffff) return COMMVQ_ERR_SHAPE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint4 *to = static_cast<uint4 *>(tables);
    k_tree_pack<<<dim3((unsigned)(kp / 256)), 256, 0, s>>>(static_cast<const uint4 *>(key_cb), to, c.m_key, kp);
    if (hipGetLastError() != hipSuccess) return COMMVQ_ERR_LAUNCH;
    k_tree_pack<<<dim3((unsigned)(vp / 256)), 256, 0, s>>>(static_cast<const uint4 *>(val_cb), to + kp, c.m_val, vp);
    if (hipGetLastError() != hipSuccess) return COMMVQ_ERR_LAUNCH;
    float *scales = reinterpret_cast<float *>(static_cast<char *>(tables) + tree_packed_bytes(c));
    k_tree_scale<<<dim3((unsigned)c.n_kv_heads), 1024, 0, s>>>(static_cast<const uint4 *>(key_cb), scales, c.m_key);
    if (hipGetLastError() != hipSuccess) return COMMVQ_ERR_LAUNCH;
    k_tree_scale<<<dim3((unsigned)c.n_kv_heads), 1024, 0, s>>>(static_cast<const uint4 *>(val_cb), scales + 1, c.m_val);
    return hipGetLastError() == hipSuccess ? COMMVQ_OK : COMMVQ_ERR_LAUNCH;
}

}  // extern "C"
