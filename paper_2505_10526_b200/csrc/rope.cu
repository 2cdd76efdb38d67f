// Rotary positions of queries and keys (massv_rotary).
//
// A CTA takes a few tokens.  It first makes the sine and cosine of every (token, pair), one per thread, and then every (token, head,
// pair group) turns with them, so the angle of a pair is computed once however many heads share it.  Nothing is lost at far positions: turns per
// position are a 64-bit fraction, and position * fraction wraps modulo 2^64 exactly where the angle wraps modulo one turn, so
// the upper bits are the angle in [-1/2, 1/2) turns (off by what the fraction was rounded by times the position, 2^-29 of a turn at most).  The heads' elements are requested ahead of that, so that
// the arithmetic of the angles runs under the loads.  HBM bounds it: one read and one write of the heads, 8,191 tokens of 28 + 4 heads
// of 128 24 us (5.5 TB/s), 32,768 97 us; a block of six tokens is a launch, 2.9 us.
#include <math.h>

#include "kernels.cuh"

namespace massv {

namespace {

constexpr int kRopeThreads = 256;
// Work items of a thread whose loads are in flight together: with pairs half a head apart an item is two loads, and four of them take the
// registers of a fourth CTA per SM (8,191 tokens of 32 heads of 128: 33.0 us with four, 24.5 with two; adjacent pairs 97 against 91).
template <bool HALF> constexpr int kRopeBatch = HALF ? 2 : 4;
constexpr int kRopeMaxPairs = 128;
constexpr int kRopeMaxTokens = 4;

template <int V> struct RopeVec;
template <> struct RopeVec<8> { using T = uint4; };
template <> struct RopeVec<2> { using T = uint32_t; };
template <> struct RopeVec<1> { using T = uint16_t; };

template <int V>
__device__ __forceinline__ void unpack(const typename RopeVec<V>::T& x, float (&f)[V]) {
    const __nv_bfloat16* h = reinterpret_cast<const __nv_bfloat16*>(&x);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = __bfloat162float(h[i]);
}
template <int V>
__device__ __forceinline__ typename RopeVec<V>::T pack(const float (&f)[V]) {
    typename RopeVec<V>::T x;
    __nv_bfloat16* h = reinterpret_cast<__nv_bfloat16*>(&x);
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = __float2bfloat16_rn(f[i]);
    return x;
}

// V: elements per access.  HALF: an item is V pairs, as V elements at i and V at i + rot_dim / 2 (V divides rot_dim / 2), or V elements
// behind rot_dim that are copied.  Interleaved: an item is 8 elements, of which those below rot_dim turn.  A thread keeps its place
// within a head and goes from (token, head) row to row, so there is nothing to divide; the angles' sines and cosines lie in shared memory such
// that neighbouring places read neighbouring words.
template <bool HALF, int V>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p) {
    using T = typename RopeVec<V>::T;
    constexpr int kPairs = HALF ? V : V / 2;             // pairs of an item
    __shared__ float2 s_cs[kRopeMaxTokens][kRopeMaxPairs + kPairs];
    const int pairs = p.rot_dim / 2, turning = HALF ? pairs / V : (p.rot_dim + V - 1) / V;
    const int units = turning + (p.copy ? (p.d - (HALF ? p.rot_dim : turning * V)) / V : 0);      // items of a head
    const int heads = p.Hq + p.Hkv;
    const long long n_tokens = (long long)p.B * p.rows, token0 = (long long)blockIdx.x * p.tokens_per_cta;
    const int n_rows = (int)min((long long)p.tokens_per_cta, n_tokens - token0) * heads;
    const int step = kRopeThreads / units, first = threadIdx.x / units, unit = threadIdx.x - first * units;      // (units <= 256)
    const bool turns = unit < turning;
    const int e = HALF && !turns ? p.rot_dim + (unit - turning) * V : unit * V;                  // the item's first element
    pdl_wait();
    pdl_trigger();

    struct Row { int tok, h; };
    auto advance = [&](Row& r) {
        r.h += step;
        while (r.h >= heads) { r.h -= heads; ++r.tok; }
    };
    auto source = [&](const Row& r) {
        const long long t = token0 + r.tok;
        return (r.h < p.Hq ? p.q + t * p.q_stride + r.h * p.d : p.k + t * p.k_stride + (r.h - p.Hq) * p.d) + e;
    };
    auto target = [&](const Row& r) {
        const long long t = token0 + r.tok;
        return (r.h < p.Hq ? p.q_out + t * p.q_out_stride + r.h * p.d : p.k_out + t * p.k_out_stride + (r.h - p.Hq) * p.d) + e;
    };
    Row row{0, first < step ? first : 0};
    while (row.h >= heads) { row.h -= heads; ++row.tok; }
    bool have_angles = false;
    for (int base = first < step ? first : n_rows; base < n_rows || !have_angles; base += step * kRopeBatch<HALF>) {
        T a[kRopeBatch<HALF>], b[kRopeBatch<HALF>];
        Row at = row;
#pragma unroll
        for (int k = 0; k < kRopeBatch<HALF>; ++k) {
            if (base + k * step < n_rows) {
                const __nv_bfloat16* src = source(at);
                a[k] = *reinterpret_cast<const T*>(src);
                if (HALF && turns) b[k] = *reinterpret_cast<const T*>(src + pairs);
                advance(at);
            }
        }
        if (!have_angles) {
            have_angles = true;
            const int n_tok = n_rows / heads;
            for (int i = threadIdx.x; i < n_tok * pairs; i += kRopeThreads) {
                const int tok = i / pairs, pair = i - tok * pairs;
                const long long t = token0 + tok;
                long long pos;
                if (p.positions) {
                    const int axis = pair < p.axis_end[0] ? 0 : pair < p.axis_end[1] ? 1 : 2;
                    pos = p.positions[t * p.n_axes + axis];
                } else {
                    const long long seq = t / p.rows;
                    pos = (long long)p.seq_lens[seq] + (p.pos_delta ? p.pos_delta[seq] : 0) + (t - seq * p.rows);
                }
                const long long phase = (long long)((unsigned long long)pos * p.turns[pair]);
                float sn, cs;
                sincospif((float)phase * 0x1p-63f, &sn, &cs);             // phase: turns * 2^64
                s_cs[tok][pair % kPairs * turning + pair / kPairs] = make_float2(cs * p.magnitude, (p.backward ? -sn : sn) * p.magnitude);
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kRopeBatch<HALF>; ++k) {
            if (base + k * step >= n_rows) break;
            T* dst = reinterpret_cast<T*>(target(row));
            const float2* cs = s_cs[row.tok] + unit;
            advance(row);
            if (!turns) { *dst = a[k]; continue; }
            float x[V];
            unpack<V>(a[k], x);
            if constexpr (HALF) {
                float y[V];
                unpack<V>(b[k], y);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float2 c = cs[i * turning];
                    const float u = x[i] * c.x - y[i] * c.y, w = x[i] * c.y + y[i] * c.x;
                    x[i] = u; y[i] = w;
                }
                *reinterpret_cast<T*>(reinterpret_cast<__nv_bfloat16*>(dst) + pairs) = pack<V>(y);
            } else {
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    if (e / 2 + i >= pairs) break;                        // the rest of the group is behind rot_dim
                    const float2 c = cs[i * turning];
                    const float u = x[2 * i] * c.x - x[2 * i + 1] * c.y, w = x[2 * i] * c.y + x[2 * i + 1] * c.x;
                    x[2 * i] = u; x[2 * i + 1] = w;
                }
            }
            *dst = pack<V>(x);
        }
    }
}

template <bool HALF, int V>
cudaError_t launch(const RopeParams& p, int grid, cudaStream_t stream) {
    return launch_pdl(rope_kernel<HALF, V>, dim3(grid), dim3(kRopeThreads), 0, stream, p);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& in, cudaStream_t stream) {
    RopeParams p = in;
    const long long tokens = (long long)p.B * p.rows;
    // several tokens to a CTA once there are enough of them to fill the machine (28 + 4 heads of 128, one token to a CTA against four: 300
    // tokens 4.45 and 4.51 us, 1,184 5.1 and 4.7, 2,400 9.1 and 7.5, 8,191 31.1 and 23.3)
    p.tokens_per_cta = tokens >= 8LL * device_sm_count() ? kRopeMaxTokens : 1;
    const int grid = (int)((tokens + p.tokens_per_cta - 1) / p.tokens_per_cta);
    const int half = p.rot_dim / 2;
    cudaError_t e;
    if (!p.half) e = launch<false, 8>(p, grid, stream);
    else if (half % 8 == 0) e = launch<true, 8>(p, grid, stream);       // (d is a multiple of 8: the tail is whole groups too)
    else if (half % 2 == 0) e = launch<true, 2>(p, grid, stream);
    else e = launch<true, 1>(p, grid, stream);
    if (e != cudaSuccess) return e;
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace massv
