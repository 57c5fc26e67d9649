// Matrix product of ciphertexts and 8-bit integer weights (he_ct_i8_mac): for every output o of a layer, modulo each limb's q,
//   out[o][c][n] = tok[n] * (s_o * sum_t w_t * x_t[c][n]) + [c = 0] b[o],
// w_t whole numbers in [-128, 127], s_o the channel's scale and tok the tokens' (one per slot, where given).
//
// A weight is one digit, so the eight bytes of a residue need not be spread over sums of their own as for plaintexts of full
// width (he_mac_digits.hip: 64 int8 products per term): with x = sum_d x_d 256^d,
//   sum_t w_t x_t = sum_d 256^d S_d,   S_d = sum_t w_t x_td,
// one int8 product per byte.  Bytes are unsigned and the matrix cores' operands signed: x_d - 128 is the byte with its top bit
// flipped, and what that leaves out, 128 sum_d 256^d sum_t w_t, is a constant of the output.
//
// v_mfma_i32_32x32x32_i8 takes 32 terms times 32 outputs times 32 slots of one digit.  A lane's share of the input operand is one byte of 16
// terms at one slot: it loads four bytes of each of the 16 residues and transposes them in registers (4 x 4 bytes: eight byte
// permutations).  A wavefront takes half of the digits (bytes 0 .. ND-1 or ND .. 2 ND-1, ND = 2, 3 or 4 by the modulus), so
// that up to 128 outputs times 32 slots of sums fit its registers and the inputs are read once for up to 128 outputs; two
// wavefronts share a slot, and meet at the end to add their parts.  Residues in packed storage are four bytes: one wavefront.
//
// The end of an output: y = sum of its digits' sums, |y| < 2^55.1, plus 2^56, is multiplied by s_o (the upper half's by s_o 256^ND) with a
// Shoup product, which reduces it and applies the channel's scale at once; the offsets, the flipped bits' constant and s_o are
// one constant per output and limb.
#include <string.h>

#include <algorithm>
#include <type_traits>
#include <unordered_map>

#include "he_internal.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef u32 u32_any __attribute__((aligned(1)));  // four bytes of a residue, at any byte

constexpr u32 THREADS = 256, WAVES = THREADS / 64;
constexpr int OFFSET_BITS = 56;  // what makes a part of a sum positive

template <typename V>
struct Form {
    static constexpr u32 PARTS = sizeof(V) / 4;               // wavefronts that share a slot
    static constexpr u32 SLOTS = 32 * WAVES / PARTS;          // slots of a workgroup
};

template <typename V>
struct I8Args {
    const I8Group* groups;
    const u32* lists;
    const v4i* table;
    const I8Mult* mult;     // [limb][n_out][2]
    const u64* addend;      // [limb][n_out]
    const V* ct_in;
    const V* token;         // [limbs][N] or null
    const u64* bias;        // [n_out][limbs] or null
    V* out;
    u32 limbs, N, n_out;
    u32 first, n_groups;
    u32 accumulate;
};

// four bytes of four terms -> the same byte of the four terms, for the first ND bytes, as signed digits
template <int ND>
__device__ __forceinline__ void transpose4(u32 a, u32 b, u32 c, u32 d, u32 (&out)[ND]) {
    const u32 lo0 = __builtin_amdgcn_perm(b, a, 0x05010400u), lo1 = __builtin_amdgcn_perm(d, c, 0x05010400u);
    out[0] = __builtin_amdgcn_perm(lo1, lo0, 0x05040100u) ^ 0x80808080u;
    out[1] = __builtin_amdgcn_perm(lo1, lo0, 0x07060302u) ^ 0x80808080u;
    if constexpr (ND > 2) {
        const u32 hi0 = __builtin_amdgcn_perm(b, a, 0x07030602u), hi1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
        out[2] = __builtin_amdgcn_perm(hi1, hi0, 0x05040100u) ^ 0x80808080u;
        if constexpr (ND > 3) out[3] = __builtin_amdgcn_perm(hi1, hi0, 0x07060302u) ^ 0x80808080u;
    }
}

// Workgroup barrier that orders LDS traffic only.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// floor(w * 2^64 / q) for w < q: the quotient estimate from the upper word of the Barrett ratio and the product with the lower
// one is short by at most 2
__device__ __forceinline__ u64 shoup_companion(u64 w, const LimbConst& c) {
    u64 e = w * c.ratio_hi + mul_hi64(w, c.ratio_lo);
    u64 r = 0 - e * c.q;  // w * 2^64 - e * q, below 4q < 2^64
#pragma unroll
    for (int i = 0; i < 3; i++) {
        const bool more = r >= c.q;
        e += more;
        r -= more ? c.q : 0;
    }
    return e;
}

template <typename V, int OT, int ND>
__device__ __forceinline__ void i8_body(const I8Args<V>& a, const LimbConst& c, const I8Group& g, u32 part, u32 row, u64* exchange) {
    const u32 lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    const u32 comp = row & 1, limb = row >> 1;
    const u32 upper = sizeof(V) == 8 ? wave & 1 : 0;         // which half of the digits
    const u32 slot = part * Form<V>::SLOTS + wave / Form<V>::PARTS * 32 + lane % 32;
    const size_t at = ((size_t)comp * a.limbs + limb) * a.N + slot;
    const u32 ct_stride = 2 * a.limbs * a.N * sizeof(V);     // bytes
    const char* x_base = reinterpret_cast<const char*>(a.ct_in + at) + upper * ND;
    const u32 blocks = (g.n_terms + 31) / 32;

    v16i sums[OT][ND];
#pragma unroll
    for (int o = 0; o < OT; o++)
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) sums[o][d][i] = 0;

    const u32* list = a.lists + (size_t)g.list * 32 + half * 16;
    const v4i* table = a.table + (size_t)g.table * 64 + lane;
    for (u32 b = 0; b < blocks; b++) {
        u32 x[16];
#pragma unroll
        for (int j = 0; j < 16; j++) x[j] = *reinterpret_cast<const u32_any*>(x_base + (u64)list[b * 32 + j] * ct_stride);
        v4i in[ND];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            u32 t[ND];
            transpose4<ND>(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3], t);
#pragma unroll
            for (int d = 0; d < ND; d++) in[d][j] = (int)t[d];
        }
#pragma unroll
        for (int o = 0; o < OT; o++) {
            const v4i w = table[(b * OT + o) * 64];
#pragma unroll
            for (int d = 0; d < ND; d++) sums[o][d] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, in[d], sums[o][d], 0, 0, 0);
        }
    }

    // the ends of the outputs: tiles of 32, of which a lane holds 16 at its slot
    u64 tok = 0, tok_shoup = 0;
    if (a.token) {
        tok = a.token[(size_t)limb * a.N + slot];
        tok_shoup = shoup_companion(tok, c);
    }
    const size_t out_stride = (size_t)2 * a.limbs * a.N;
    auto store = [&](u32 o, u64 v) {  // v < 4q, congruent to the scaled sum without the addend
        v = v >= c.two_q ? v - c.two_q : v;
        v += a.addend[(size_t)limb * a.n_out + g.out0 + o];
        v = v >= c.two_q ? v - c.two_q : v;
        v = v >= c.q ? v - c.q : v;
        if (a.token) v = shoup_mul(v, tok, tok_shoup, c.q);
        if (a.bias && comp == 0) v = add_mod(v, a.bias[(size_t)(g.out0 + o) * a.limbs + limb], c.q);
        V* dst = a.out + (g.out0 + o) * out_stride + at;
        if (a.accumulate) v = add_mod(v, *dst, c.q);
        *dst = (V)v;
    };
    // this lane's output r (0 .. 15) of tile o, and its part of the sum, below 2q
    auto output_of = [&](int o, int r) -> u32 { return 32 * o + 8 * (r / 4) + 4 * half + r % 4; };
    auto part_of = [&](int o, int r) -> u64 {
        const u32 mine = min(output_of(o, r), g.count - 1);
        const I8Mult m = a.mult[((size_t)limb * a.n_out + g.out0 + mine) * 2 + upper];
        int64_t y = 1ll << OFFSET_BITS;
#pragma unroll
        for (int d = 0; d < ND; d++) y += (int64_t)sums[o][d][r] << (8 * d);
        return shoup_mul_lazy((u64)y, m.w, m.w_shoup, c.q);
    };
    if constexpr (sizeof(V) == 8) {
        // of every tile the wavefront of the lower digits finishes the first eight of a lane's outputs, the other one the last eight
        auto finish = [&](auto of_upper) {
            constexpr int KEEP = decltype(of_upper)::value ? 8 : 0, SEND = 8 - KEEP;
#pragma unroll
            for (int o = 0; o < OT; o++) {
                if (32 * (u32)o >= g.count) break;
                u64* buf = exchange + (o & 1) * (WAVES * 8 * 64) + lane;
#pragma unroll
                for (int k = 0; k < 8; k++) buf[(wave * 8 + k) * 64] = part_of(o, SEND + k);
                lds_barrier();
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    const u64 v = part_of(o, KEEP + k) + buf[((wave ^ 1) * 8 + k) * 64];
                    if (output_of(o, KEEP + k) < g.count) store(output_of(o, KEEP + k), v);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        if (upper) finish(std::true_type{});
        else finish(std::false_type{});
    } else {
#pragma unroll
        for (int o = 0; o < OT; o++) {
            if (32 * (u32)o >= g.count) break;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const u64 v = part_of(o, r);
                if (output_of(o, r) < g.count) store(output_of(o, r), v);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
}

template <typename V, int OT>
__global__ void __launch_bounds__(THREADS, OT == 1 ? 3 : OT == 2 ? 2 : 1) i8_mac_kernel(LimbTable lt, I8Nd nd, I8Args<V> a) {
    __shared__ u64 exchange[sizeof(V) == 8 ? 2 * WAVES * 8 * 64 : 1];
    // Workgroups go to the eight XCDs round-robin: the eight slices of a run of slots fastest, then the groups, so that the groups
    // that read one slice run on one XCD, close in time, and find its inputs in that L2.
    const u32 parts8 = a.N / Form<V>::SLOTS / 8;
    u32 b = blockIdx.x / 8;
    const u32 group = b % a.n_groups;
    b /= a.n_groups;
    const u32 part = b % parts8 * 8 + blockIdx.x % 8, row = b / parts8;
    const I8Group g = a.groups[a.first + group];
    const LimbConst& c = lt.c[row >> 1];
    const u32 digits = sizeof(V) == 8 ? nd.nd[row >> 1] : 4;
    if (digits == 4) i8_body<V, OT, 4>(a, c, g, part, row, exchange);
    else if constexpr (sizeof(V) == 8) {
        if (digits == 3) i8_body<V, OT, 3>(a, c, g, part, row, exchange);
        else i8_body<V, OT, 2>(a, c, g, part, row, exchange);
    }
}

template <typename V>
u64 class_blocks(const he_ctx* ctx, const he_i8_layer* l, u32 limbs, u32 cls) {
    return (u64)(l->class_begin[cls + 1] - l->class_begin[cls]) * (ctx->N / Form<V>::SLOTS) * 2 * limbs;
}

template <typename V, int OT>
int launch_class(he_ctx* ctx, I8Args<V> a, const he_i8_layer* l, hipStream_t s) {
    a.first = l->class_begin[OT - 1];
    a.n_groups = l->class_begin[OT] - a.first;
    if (a.n_groups == 0) return HE_OK;
    hipLaunchKernelGGL((i8_mac_kernel<V, OT>), dim3((u32)class_blocks<V>(ctx, l, a.limbs, OT - 1)), dim3(THREADS), 0, s, ctx->limbs, l->nd, a);
    HE_HIP(hipGetLastError());
    return HE_OK;
}

template <typename V>
int launch(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const V* ct_in, const V* token, const u64* bias, V* out, u32 accumulate, hipStream_t s) {
    const I8Args<V> a{l->groups_dev, l->lists_dev, reinterpret_cast<const v4i*>(l->table_dev), l->mult_dev, sizeof(V) == 8 ? l->addend_dev : l->addend32_dev,
                      ct_in, token, bias, out, limbs, ctx->N, l->n_out, 0, 0, accumulate};
    int rc;
    if ((rc = launch_class<V, 1>(ctx, a, l, s)) != HE_OK) return rc;
    if ((rc = launch_class<V, 2>(ctx, a, l, s)) != HE_OK) return rc;
    if ((rc = launch_class<V, 3>(ctx, a, l, s)) != HE_OK) return rc;
    return launch_class<V, 4>(ctx, a, l, s);
}

u64 mul_mod_host(u64 a, u64 b, u64 q) { return (u64)((u128)a * b % q); }

// the terms of an output: where they start
struct Rows {
    const u32 *off, *ct, *pt;
    u32 terms(u32 o) const { return off[o + 1] - off[o]; }
    bool same_inputs(u32 a, u32 b) const {
        return terms(a) == terms(b) && (terms(a) == 0 || memcmp(ct + off[a], ct + off[b], (size_t)terms(a) * 4) == 0);
    }
};

}  // namespace

// every launch of a call must fit a grid
int check_i8_launch(he_ctx* ctx, const he_i8_layer* l, u32 limbs, bool packed) {
    for (u32 cls = 0; cls < I8_CLASSES; cls++)
        if ((packed ? class_blocks<u32>(ctx, l, limbs, cls) : class_blocks<u64>(ctx, l, limbs, cls)) > 0x7FFFFFFFull) return HE_ERR_RANGE;
    return HE_OK;
}

// The host's part of a layer: groups, lists, table and constants (throws std::bad_alloc).
void build_i8_layer(const he_ctx* ctx, const u32* off, const u32* term_ct, const u32* term_pt, const int8_t* weights, const u64* scale,
                    he_i8_layer* l, I8Host& h) {
    const Rows rows{off, term_ct, term_pt};
    const u32 n_out = l->n_out;
    // Runs of outputs that read the same inputs in the same order, cut into groups of up to 128 with the same number of tiles.
    std::vector<I8Group> classes[I8_CLASSES];
    std::unordered_multimap<u64, I8Group> known;  // groups by a hash of their weights, to share tables
    for (u32 o = 0; o < n_out;) {
        u32 end = o + 1;
        while (end < n_out && rows.same_inputs(o, end)) end++;
        const u32 tiles = (end - o + 31) / 32, cuts = (tiles + I8_CLASSES - 1) / I8_CLASSES, per = (tiles + cuts - 1) / cuts;
        const u32 terms = rows.terms(o), blocks = (terms + 31) / 32;
        const u32 list = (u32)(h.lists.size() / 32);
        for (u32 t = 0; t < blocks * 32; t++) h.lists.push_back(term_ct[off[o] + std::min(t, terms - 1)]);
        for (; o < end; o += std::min(per * 32, end - o)) {
            I8Group g{o, std::min(per * 32, end - o), terms, list, 0, {0, 0, 0}};
            const size_t n = (size_t)g.count * terms;  // the plaintexts of a group's outputs follow one another
            u64 hash = 0xCBF29CE484222325ull ^ n;
            for (size_t i = 0; i < n; i++) hash = (hash ^ term_pt[off[o] + i]) * 0x100000001B3ull;
            bool found = false;
            const auto range = known.equal_range(hash);
            for (auto it = range.first; it != range.second && !found; ++it) {
                const I8Group& k = it->second;
                if (k.count != g.count || k.n_terms != terms || (n && memcmp(term_pt + off[k.out0], term_pt + off[o], n * 4) != 0)) continue;
                g.table = k.table;
                found = true;
            }
            if (!found) {
                // [block][tile][lane][16]: row lane % 32 of the tile, terms 16 * (lane / 32) .. of the block
                g.table = (u32)(h.table.size() / 1024);
                h.table.resize(h.table.size() + (size_t)blocks * per * 1024, 0);
                int8_t* t0 = h.table.data() + (size_t)g.table * 1024;
                for (u32 r = 0; r < g.count; r++)
                    for (u32 t = 0; t < terms; t++)
                        t0[(((size_t)t / 32 * per + r / 32) * 64 + t % 32 / 16 * 32 + r % 32) * 16 + t % 16] = weights[term_pt[off[o + r] + t]];
                known.emplace(hash, g);
            }
            classes[per - 1].push_back(g);
        }
    }
    for (u32 cls = 0; cls < I8_CLASSES; cls++) {
        l->class_begin[cls] = (u32)h.groups.size();
        h.groups.insert(h.groups.end(), classes[cls].begin(), classes[cls].end());
    }
    l->class_begin[I8_CLASSES] = (u32)h.groups.size();
    // Per limb and output: the multipliers of the two halves of a sum and the constant that goes with them.
    std::vector<int64_t> weight_sum(n_out);
    for (u32 o = 0; o < n_out; o++)
        for (u32 t = off[o]; t < off[o + 1]; t++) weight_sum[o] += weights[term_pt[t]];
    h.mult.resize((size_t)ctx->L * n_out * 2);
    h.addend.resize((size_t)ctx->L * n_out);
    h.addend32.resize((size_t)ctx->L * n_out);
    for (u32 i = 0; i < ctx->L; i++) {
        const u64 q = ctx->q[i];
        u32 bits = 0;
        while (q >> bits) bits++;
        const u32 nd = std::max<u32>(2, ((bits + 7) / 8 + 1) / 2);
        l->nd.nd[i] = nd;
        const u64 shift = (u64)(((u128)1 << (8 * nd)) % q), offset = (1ull << OFFSET_BITS) % q;
        u64 flipped = 0, flipped32 = 0;  // what the digits' top bits stand for, all 2 nd of them, and four
        for (u32 d = 0; d < 2 * nd; d++) flipped |= 0x80ull << (8 * d);
        flipped32 = 0x80808080u % q;
        flipped %= q;
        for (u32 o = 0; o < n_out; o++) {
            const size_t k = (size_t)i * n_out + o;
            const u64 s = scale ? scale[(size_t)o * ctx->L + i] : 1 % q, t = mul_mod_host(s, shift, q);
            h.mult[2 * k] = I8Mult{s, (u64)(((u128)s << 64) / q)};
            h.mult[2 * k + 1] = I8Mult{t, (u64)(((u128)t << 64) / q)};
            const u64 sum = (u64)(((__int128)weight_sum[o] % (__int128)q + q) % q);
            const u64 both = (u64)(((u128)offset + mul_mod_host(offset, shift, q)) % q);
            h.addend[k] = mul_mod_host(s, (mul_mod_host(flipped, sum, q) + q - both) % q, q);
            h.addend32[k] = mul_mod_host(s, (mul_mod_host(flipped32, sum, q) + q - offset) % q, q);
        }
    }
}

int launch_i8(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const u64* ct_in, const u64* token, const u64* bias, u64* out, u32 accumulate,
              hipStream_t s) {
    return launch<u64>(ctx, l, limbs, ct_in, token, bias, out, accumulate, s);
}

int launch_i8_32(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const u32* ct_in, const u32* token, const u64* bias, u32* out, u32 accumulate,
                 hipStream_t s) {
    return launch<u32>(ctx, l, limbs, ct_in, token, bias, out, accumulate, s);
}
