// Rules on logits (massv_logits_apply, massv_accept_logits) and the token history they read (massv_history_add).
//
// One warp takes 1,024 logits of one row, 8 x 4 per lane, all requested at once; the rows of a sequence sit in one CTA, which shares
// what belongs to the sequence (its biases).  Nearly every token is under no rule but the grammar's bit: what marks the others is one
// bit per token (prompt, output, draft, bias), 32 words per slice, one per lane.  The marked tokens are
// listed, worked out by 32 lanes at a time, with the counts only they need, and left in shared memory, where the owners of those logits pick
// them up.  (Each lane on the marks of its own word takes up to 32 turns where frequent tokens have low numbers: 16 rows of 152,064
// 15.5 us against 10.1.)  So the pass costs one read and one write of the logits and a bit per token and mask.  What
// bounds it is latency at the occupancy it has: a CTA asks for its masks, then for the logits they allow, then for the counts of marked tokens, with 3 or 4 CTAs
// to an SM (72 registers with statistics) or 2 (83 KB of shared memory with biases and one row per sequence); 64 x 8 rows of 262,144
// with 2 % allowed 215 us, where the bytes it moves take 130.  With statistics (for the acceptance) the same
// pass leaves maximum, sum of exponentials and argmax of its 1,024 logits as one partial slot of the row.
#include "kernels.cuh"

namespace massv {

namespace {

constexpr int kWords = kLogitSlice / 32;         // mask words of a slice
constexpr int kVecs = kLogitSlice / 128;         // groups of four logits per lane
static_assert(kWords == 32, "one mask word per lane");
constexpr int kMaxWarps = 8;

// VEC4: rows start on 16-byte boundaries (V is a multiple of 4) and a group of four lies inside the row or outside it.
template <bool VEC4, bool STATS>
__global__ void __launch_bounds__(kMaxWarps * 32) logit_rules_kernel(const LogitsParams p, int slices_per_cta) {
    extern __shared__ float s_dyn[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int local = warp / p.R, j = warp % p.R;                 // slice within the CTA, row within the sequence
    const int b = blockIdx.y, slice0 = blockIdx.x * slices_per_cta, slice = slice0 + local;
    const int v0 = slice * kLogitSlice, W = (p.V + 31) / 32;
    float* adj = s_dyn + warp * (kLogitSlice + kLogitSlice / 2);   // logits of the marked tokens, by position in the slice
    uint16_t* list = reinterpret_cast<uint16_t*>(adj + kLogitSlice);       // their positions
    int* slot = reinterpret_cast<int*>(s_dyn + (blockDim.x >> 5) * (kLogitSlice + kLogitSlice / 2));      // [slices_per_cta][1024]: the token's last bias entry, -1: none
    uint32_t* bias_bits = reinterpret_cast<uint32_t*>(slot + slices_per_cta * kLogitSlice);
    pdl_wait();
    pdl_trigger();

    if (p.repetition && blockIdx.x == 0 && threadIdx.x == 0 && !(p.repetition[b] > 0.f)) set_status(p.dev_status, MASSV_ERR_INVALID_ARG);

    // ---- what the masks say, then the logits of allowed tokens, all requested ahead of what follows
    const size_t row = (size_t)b * p.R + j;
    const float* z = p.logits + row * p.V + v0;
    const int valid = max(0, min(kLogitSlice, p.V - v0));          // (none: past the last slice)
    const int word = v0 / 32 + lane;
    const bool has_word = word < W;
    const uint32_t allowed = p.allowed && has_word ? p.allowed[row * W + word] : 0xffffffffu;
    const uint32_t prompt = p.prompt_bits && has_word ? p.prompt_bits[(size_t)b * W + word] : 0u;
    const uint32_t output = p.output_bits && has_word ? p.output_bits[(size_t)b * W + word] : 0u;
    int k0 = p.bias_start ? p.bias_start[b] : 0, k1 = p.bias_start ? p.bias_start[b + 1] : 0;
    // The bits of this lane's groups of four, a nibble each, from a word per lane.
    auto nibbles = [&](uint32_t words) {
        uint32_t r = 0u;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) r |= (__shfl_sync(0xffffffffu, words, k * 4 + lane / 8) >> (lane % 8 * 4) & 15u) << (4 * k);
        return r;
    };
    const uint32_t may = p.allowed ? nibbles(allowed) : 0xffffffffu;
    float x[kVecs][4];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const uint32_t nib = may >> (4 * k) & 15u;
        const int e0 = k * 128 + lane * 4;
        if constexpr (VEC4) {
            float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (nib && e0 < valid) v = *reinterpret_cast<const float4*>(z + e0);
            x[k][0] = v.x; x[k][1] = v.y; x[k][2] = v.z; x[k][3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[k][e] = nib >> e & 1u && e0 + e < valid ? z[e0 + e] : -INFINITY;
        }
    }

    // ---- the sequence's biases that fall into this CTA's slices
    int bias_n = 0;
    if (p.bias_start) {
        if (k0 < 0 || k1 < k0 || k1 > p.n_bias) {
            if (blockIdx.x == 0 && threadIdx.x == 0) set_status(p.dev_status, MASSV_ERR_INVALID_ARG);
            k0 = max(0, min(k0, p.n_bias)); k1 = max(k0, min(k1, p.n_bias));
        }
        bias_n = k1 - k0;
        if (bias_n > 0) {
            for (int i = threadIdx.x; i < slices_per_cta * kLogitSlice; i += blockDim.x) slot[i] = -1;
            for (int i = threadIdx.x; i < slices_per_cta * kWords; i += blockDim.x) bias_bits[i] = 0u;
            __syncthreads();
            for (int k = k0 + (int)threadIdx.x; k < k1; k += blockDim.x) {
                const int t = p.bias_tokens[k], at = t - slice0 * kLogitSlice;
                if (t < 0 || t >= p.V) {
                    if (blockIdx.x == 0) set_status(p.dev_status, MASSV_ERR_INVALID_ARG);
                } else if (at >= 0 && at < slices_per_cta * kLogitSlice) {
                    atomicMax(&slot[at], k);                       // the last entry of a token counts, in whatever order they come here
                    atomicOr(&bias_bits[at / 32], 1u << (at % 32));
                }
            }
            __syncthreads();
        }
    }
    if (valid == 0) return;                                        // (no barrier behind this)

    // ---- the marked tokens
    const uint32_t biased = bias_n > 0 ? bias_bits[local * kWords + lane] : 0u;
    uint32_t drafted = 0u;
    if (p.drafts)
        for (int i = 0; i < j; ++i) {                              // the row follows the drafts ahead of it
            const int d = p.drafts[(size_t)b * (p.R - 1) + i];
            if (d >= 0 && d < p.V && d / 32 == word) drafted |= 1u << (d % 32);
        }
    const uint32_t marked = (prompt | output | biased | drafted) & allowed & (lane * 32 + 32 <= valid ? 0xffffffffu : lane * 32 < valid ? (1u << (valid - lane * 32)) - 1u : 0u);
    uint32_t changes = 0u;
    if (__any_sync(0xffffffffu, marked != 0u)) {
        changes = nibbles(marked);
        float rep = p.repetition ? p.repetition[b] : 1.f;
        if (!(rep > 0.f)) rep = 1.f;
        const float freq = p.frequency ? p.frequency[b] : 0.f, pres = p.presence ? p.presence[b] : 0.f;
        const int mine = __popc(marked);
        int at_end = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, at_end, o);
            if (lane >= o) at_end += v;
        }
        const int n = __shfl_sync(0xffffffffu, at_end, 31);
        int at_list = at_end - mine;
        for (uint32_t rest = marked; rest; rest &= rest - 1) list[at_list++] = (uint16_t)(lane * 32 + __ffs(rest) - 1);
        __syncwarp();
#pragma unroll 2
        for (int i0 = 0; i0 < n; i0 += 32) {
            const bool have = i0 + lane < n;
            const int at = have ? list[i0 + lane] : 0, from = at >> 5, bit = at & 31;
            const uint32_t pr = __shfl_sync(0xffffffffu, prompt, from) >> bit, ou = __shfl_sync(0xffffffffu, output, from) >> bit,
                           bi = __shfl_sync(0xffffffffu, biased, from) >> bit, dr = __shfl_sync(0xffffffffu, drafted, from) >> bit;
            if (have) {
                int c = ou & 1u ? p.counts[(size_t)b * p.V + v0 + at] : 0;
                float t = z[at];
                const float bias = bi & 1u ? p.bias_values[slot[local * kLogitSlice + at]] : 0.f;
                if (dr & 1u)
                    for (int i = 0; i < j; ++i) c += p.drafts[(size_t)b * (p.R - 1) + i] == v0 + at ? 1 : 0;
                // each operation rounded by itself, never contracted
                if (bi & 1u) t = __fadd_rn(t, bias);
                if (p.repetition && ((pr & 1u) || c > 0)) t = t > 0.f ? __fdiv_rn(t, rep) : __fmul_rn(t, rep);
                if (p.frequency && c > 0) t = __fsub_rn(t, __fmul_rn(freq, (float)c));
                if (p.presence && c > 0) t = __fsub_rn(t, pres);
                adj[at] = t;
            }
        }
        __syncwarp();
    }

    // ---- every logit as the rules leave it; out
    float* out = p.out ? p.out + row * p.V + v0 : nullptr;
    const bool in_place = p.out == p.logits;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
        const int e0 = k * 128 + lane * 4;
        const uint32_t m = changes >> (4 * k) & 15u, a = may >> (4 * k) & 15u;
        if (a != 15u) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(a >> e & 1u)) x[k][e] = -INFINITY;
        }
        if (m) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (m >> e & 1u) x[k][e] = adj[e0 + e];
        }
        if (out && !(in_place && m == 0u && a == 15u)) {
            if constexpr (VEC4) {
                if (e0 < valid) *reinterpret_cast<float4*>(out + e0) = make_float4(x[k][0], x[k][1], x[k][2], x[k][3]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e0 + e < valid) out[e0 + e] = x[k][e];
            }
        }
    }

    if constexpr (STATS) {
        // (elements past the end of the row are -inf: they have no part in either)
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < kVecs; ++k) m = fmaxf(m, fmaxf(fmaxf(x[k][0], x[k][1]), fmaxf(x[k][2], x[k][3])));
        {
            // (a lane's maximum is no NaN: as a whole number that orders like it, one instruction finds the warp's)
            const int bits = __float_as_int(m), key = __reduce_max_sync(0xffffffffu, bits < 0 ? bits ^ 0x7fffffff : bits);
            m = __int_as_float(key < 0 ? key ^ 0x7fffffff : key);
        }
        float sum = 0.f;
        int idx = 0x7fffffff;
        if (m != -INFINITY) {
            if (p.greedy) {
#pragma unroll
                for (int k = kVecs - 1; k >= 0; --k) {
#pragma unroll
                    for (int e = 3; e >= 0; --e)
                        if (x[k][e] == m) idx = v0 + k * 128 + lane * 4 + e;
                }
                idx = __reduce_min_sync(0xffffffffu, idx);
            } else {
                // exp((z - max) / T) as 2^((z - max) log2(e) / T): the difference is formed before the factor rounds it
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < kVecs; ++k) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[e] += ex2_ftz((x[k][e] - m) * p.inv_T_log2e);
                }
                sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            }
        }
        if (lane == 0) {
            const size_t at = (size_t)slice * p.B * p.R + row;
            p.part_max[at] = m;
            p.part_sum[at] = sum;
            p.part_idx[at] = idx;
        }
    }
}

__global__ void __launch_bounds__(256) history_add_kernel(int B, int V, const int32_t* tokens, int n_max, const int32_t* lens, uint32_t* bits, int32_t* counts,
                                                          int32_t* dev_status) {
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    pdl_wait();
    pdl_trigger();
    const int per = max(n_max, 1);                                // (without tokens: a thread a sequence, for its length)
    if (i >= (long long)B * per) return;
    const int b = (int)(i / per), k = (int)(i % per);
    if (lens) {
        const int n = lens[b];
        if (k == 0 && (n < 0 || n > n_max)) set_status(dev_status, MASSV_ERR_INVALID_ARG);
        if (k >= min(n, n_max)) return;
    }
    const int t = tokens[i];
    if (t < 0 || t >= V) { set_status(dev_status, MASSV_ERR_INVALID_ARG); return; }
    // (sums of integers: the order of arrival does not show)
    atomicOr(bits + (size_t)b * ((V + 31) / 32) + t / 32, 1u << (t % 32));
    if (counts) atomicAdd(counts + (size_t)b * V + t, 1);
}

template <bool VEC4, bool STATS>
cudaError_t launch(const LogitsParams& p, cudaStream_t stream) {
    const int slices = logit_slices(p.V), per = p.R >= kMaxWarps ? 1 : kMaxWarps / p.R < slices ? kMaxWarps / p.R : slices, warps = per * p.R;
    const size_t smem = ((size_t)warps * (kLogitSlice + kLogitSlice / 2) + (p.bias_start ? (size_t)per * (kLogitSlice + kWords) : 0)) * 4;
    constexpr int kMaxSmem = kMaxWarps * (2 * kLogitSlice + kLogitSlice / 2 + kWords) * 4;
    const cudaError_t e = cudaFuncSetAttribute(logit_rules_kernel<VEC4, STATS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl(logit_rules_kernel<VEC4, STATS>, dim3((slices + per - 1) / per, p.B), dim3(warps * 32), smem, stream, p, per);
}

}  // namespace

int logit_slices(int V) { return (V + kLogitSlice - 1) / kLogitSlice; }

cudaError_t launch_logit_rules(const LogitsParams& p, cudaStream_t stream) {
    const bool vec4 = p.V % 4 == 0, stats = p.part_max != nullptr;
    // (the acceptance, which alone takes statistics, has vocabularies of whole groups of eight)
    const cudaError_t e = stats ? launch<true, true>(p, stream) : vec4 ? launch<true, false>(p, stream) : launch<false, false>(p, stream);
    if (e != cudaSuccess) return e;
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_history_add(int B, int V, const int32_t* tokens, int n_max, const int32_t* lens, uint32_t* bits, int32_t* counts,
                               int32_t* dev_status, cudaStream_t stream) {
    if (n_max == 0 && !lens) return cudaSuccess;                  // nothing to add and nothing to report
    const long long n = (long long)B * (n_max > 0 ? n_max : 1);
    const cudaError_t e = launch_pdl(history_add_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, B, V, tokens, n_max, lens, bits, counts, dev_status);
    if (e != cudaSuccess) return e;
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace massv
