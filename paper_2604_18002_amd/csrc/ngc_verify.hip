// Verification of drafted tokens against the target's probabilities, from given random numbers, on gfx950.
//
// The walk starts at node 0 (the pending token).  At a node the children are tried in ascending order; with S = 1, c = 0
//   drafts sampled from q:   accept x if  u S q(x) < r(x),  r = max(p - c q, 0);   else c += S, S = sum_t max(p_t - c q_t, 0)
//   drafts chosen (no q):    accept x if  u S < r(x),  r = p without the tokens already refused;   else S -= r(x)
// and where nobody is accepted the next token is drawn from r by its cumulative sums.  (A refusal leaves r <- max(r - S q, 0)
// with sum S: applied again and again that is p less one growing multiple of q, because a token that has reached 0 stays
// there; so a node's residual is one number, c, and costs no memory.)
//
// Everything the walk compares is gathered at once, a node per lane, and the walk itself is a few scalar steps per node.
// What costs is the one row (two with q) that the next token is drawn from: V floats a sequence.  S workgroups share it, in
// chunks of 1024 values whose 64-bit sums they leave in the workspace; the one that takes the last ticket adds the chunks
// up, finds the one that the random number falls into and reads it again.  A second refusal at a node that drafted by
// sampling needs the whole residual's sum before the walk can go on: every workgroup makes that for itself.
//
// Microseconds (HIP graph): one chain of 5 over 32000 tokens 7.5, 64 chains of 6 over 128000 16.5, 128 trees of 20 over 50001 13.9.
// Of the 16.5: launch 2.6, gathers and walk 1.1, the rows 8.4 (66 MB, 7.8 TB/s: part of them come from the last-level cache),
// sums and ticket 1.3, the last workgroup's reading, search and store 3.1.  Measured and not kept: 512 or 1024 threads, half
// or twice as many workgroups (0.99-1.37), the chunks' sums held in LDS (1.00-1.08).
//
// All sums are in 64 bits: a cumulative sum of 32-bit numbers in 32 bits would move the borders between tokens by more than
// a rare token is wide.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ngc.h"
#include "ngc_device.h"
#include "ngc_workspace.h"

namespace ngc {

constexpr int VF_THREADS = 256;
constexpr int VF_WAVES = VF_THREADS / NGC_WAVE;
constexpr int VF_CHUNK = 1024;              // values per chunk: 16 per lane of a wave
constexpr int VF_FIRST_TICKET = 8;          // status words [8, 62) hold tickets, a byte each: zero between launches
constexpr int VF_TICKETS = (NGC_STATUS_WORDS - 2 - VF_FIRST_TICKET) * 4;

struct VerifyArgs {
    const float *target;                    // [B][W][stride]
    const float *draft;                     // or nullptr
    const int32_t *token, *parent;          // [B][W]
    const int32_t *n_draft;                 // [B] or nullptr
    const float *u_accept, *u_sample;       // [B][W], [B]
    int32_t *path, *n_path, *next;          // [B][W], [B], [B]
    int32_t *status;
    double *sums;                           // [B][chunks], zero again at the end
    int64_t stride;
    int W, V, S, chunks;
};

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));    // rows begin at any multiple of 4 bytes

// (A q below 0 or NaN counts as 0, as such a p does.)
__device__ __forceinline__ double residual(float p, float q, double c)
{
    return __builtin_fmax((double)p - c * (double)__builtin_fmaxf(q, 0.f), 0.0);
}

// Sum over this lane and those below it.
__device__ __forceinline__ double wave_incl_scan_d(double v)
{
    const int lane = lane_id();
#pragma unroll
    for (int d = 1; d < NGC_WAVE; d *= 2) {
        const double w = __shfl_up(v, d);
        if (lane >= d) v += w;
    }
    return v;
}

// The residual of one node: what the next token is drawn from.
struct Residual {
    const float *p, *q;                     // q: nullptr unless c != 0
    double c;
    int refused;                            // this lane's: a token that counts nothing, -1: none
    int V;

    // Values first .. first + 3, 0 beyond the row.
    __device__ __forceinline__ void four(int first, double (&r)[4]) const
    {
        float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
        if (first + 4 <= V) {
            const f32x4_any a = *reinterpret_cast<const f32x4_any *>(p + first);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = a[e];
            if (q) {
                const f32x4_any b = *reinterpret_cast<const f32x4_any *>(q + first);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = b[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (first + e < V) {
                    x[e] = p[first + e];
                    if (q) y[e] = q[first + e];
                }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = residual(x[e], y[e], c);
    }
    // Takes the refused tokens out of values first .. first + 3 (of every lane; all of them lie in `chunk`).  Whole wave.
    __device__ __forceinline__ void refuse(int chunk, int first, double (&r)[4]) const
    {
        uint64_t inside = __ballot(refused >= 0 && refused / VF_CHUNK == chunk);
        while (inside) {
            const int x = __builtin_amdgcn_readlane(refused, __builtin_ctzll(inside));
            inside &= inside - 1;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = first + e == x ? 0.0 : r[e];
        }
    }
    // Sum of a chunk, by a wave, in a fixed order.
    __device__ __forceinline__ double chunk_sum(int chunk) const
    {
        double sum = 0.0;
        double r[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) four(chunk * VF_CHUNK + j * 256 + lane_id() * 4, r[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            refuse(chunk, chunk * VF_CHUNK + j * 256 + lane_id() * 4, r[j]);
            sum += (r[j][0] + r[j][1]) + (r[j][2] + r[j][3]);
        }
        return wave_sum_d(sum);
    }
};

// Sums that cross workgroups, and the L2 caches of different XCDs: device scope.
__device__ __forceinline__ void put(double *at, double v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double get(const double *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// First value of the row whose cumulative sum exceeds u * total, -1 if nothing in the row is positive.  One wave.
__device__ __forceinline__ int draw_token(const Residual &res, const double *sums, int chunks, double u)
{
    const int lane = lane_id();
    const int per = (chunks + NGC_WAVE - 1) / NGC_WAVE;
    double mine = 0.0;
    for (int i = lane * per; i < (lane + 1) * per && i < chunks; ++i) mine += get(sums + i);
    const double upto = wave_incl_scan_d(mine);
    const double total = __shfl(upto, NGC_WAVE - 1);
    if (!(total > 0.0)) return -1;
    const double x = u * total;
    // the lane, then the chunk; rounding may leave nothing above x: then the last chunk that holds anything
    const uint64_t above = __ballot(upto > x && mine > 0.0), some = __ballot(mine > 0.0);
    if (!some) return -1;
    const int owner = above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some);
    int chunk;
    double base;                            // cumulative sum in front of that chunk
    {
        const double below = __shfl(upto, owner > 0 ? owner - 1 : 0);
        double run = owner > 0 ? below : 0.0;
        int found = -1, last = -1;
        double found_base = 0.0, last_base = 0.0;
        for (int i = owner * per; i < (owner + 1) * per && i < chunks; ++i) {       // uniform
            const double s = get(sums + i);
            if (s > 0.0) { last = i; last_base = run; }
            if (found < 0 && s > 0.0 && run + s > x) { found = i; found_base = run; }
            run += s;
        }
        chunk = found >= 0 ? found : last;
        base = found >= 0 ? found_base : last_base;
    }
    // 16 consecutive values per lane
    double r[4][4], here = 0.0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int first = chunk * VF_CHUNK + lane * 16 + j * 4;
        res.four(first, r[j]);
        res.refuse(chunk, first, r[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) here += r[j][e];
    }
    const double incl = wave_incl_scan_d(here);
    const double before = __shfl_up(incl, 1);
    double run = base + (lane > 0 ? before : 0.0);
    int found = -1, last = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            run += r[j][e];
            const int at = chunk * VF_CHUNK + lane * 16 + j * 4 + e;
            if (r[j][e] > 0.0) {
                last = at;
                if (found < 0 && run > x) found = at;
            }
        }
    const uint64_t hit = __ballot(found >= 0), any = __ballot(last >= 0);
    if (hit) return __builtin_amdgcn_readlane(found, __builtin_ctzll(hit));
    return any ? __builtin_amdgcn_readlane(last, 63 - __builtin_clzll(any)) : -1;
}

__global__ __launch_bounds__(VF_THREADS) void verify_kernel(VerifyArgs a)
{
    __shared__ double wave_part[VF_WAVES];
    __shared__ double at_c;
    __shared__ int at_node, need_sum, is_last;
    __shared__ uint64_t at_refused;
    const int b = (int)blockIdx.x, share = (int)blockIdx.y;
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const int W = a.W, V = a.V;
    const bool counts = share == 0 && wv == 0;

    // A node per lane (every wave for itself: the refused tokens are looked up by lane later on); asked for together.
    const size_t at_lane = (size_t)b * W + (lane < W ? lane : W - 1);
    int nd = a.n_draft ? a.n_draft[b] : W;
    int up = a.parent[at_lane], token = a.token[at_lane];
    const float u = a.u_accept[at_lane];
    const double us = (double)a.u_sample[b];
    if (nd < 0 || nd > W) {
        if (counts && lane == 0) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], 1);
        nd = nd < 0 ? 0 : W;
    }
    int32_t *path = a.path + (size_t)b * W;
    if (nd == 0) {
        if (counts) {
            if (lane < W) path[lane] = -1;
            if (lane == 0) { a.n_path[b] = 0; a.next[b] = -1; }
        }
        return;
    }
    const float *target = a.target + (size_t)b * W * a.stride;
    const float *draft = a.draft ? a.draft + (size_t)b * W * a.stride : nullptr;

    if (lane >= nd) up = token = -1;
    const bool bad = lane < nd && (up < -1 || up >= lane || (lane > 0 && (token < 0 || token >= V)));
    const uint64_t bad_nodes = __ballot(bad);
    if (counts && lane == 0 && bad_nodes) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], __popcll(bad_nodes));
    if (bad) up = -1;                      // never reached
    float pv = 0.f, qv = 0.f;
    if (wv == 0 && up >= 0) {
        pv = target[(size_t)up * a.stride + token];
        if (draft) qv = draft[(size_t)up * a.stride + token];
    }

    // ---- the walk: wave 0; the whole workgroup where a residual's sum is wanted -------
    int node = 0, count = 1;
    double S = 1.0, c = 0.0;
    uint64_t left = 0, refused = 0;        // children of `node` not yet tried; tried
    if (wv == 0) {
        if (lane < W) path[lane] = lane == 0 ? 0 : -1;      // (every workgroup of the sequence writes the same)
        left = __ballot(up == 0);
    }
    while (true) {
        if (wv == 0) {
            bool sum = false;
            while (left) {
                const int x = __builtin_ctzll(left);
                left &= left - 1;
                const double p = (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pv), x));
                const double ux = (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(u), x));
                bool take;
                double r;
                if (draft) {
                    const double q = (double)__builtin_fmaxf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(qv), x)), 0.f);
                    r = __builtin_fmax(p - c * q, 0.0);
                    take = ux * S * q < r;
                } else {
                    const int tx = __builtin_amdgcn_readlane(token, x);
                    const bool again = (__ballot(token == tx) & refused) != 0;
                    r = again ? 0.0 : __builtin_fmax(p, 0.0);
                    take = ux * S < r;
                }
                if (take) {
                    node = x;
                    if (lane == 0) path[count] = x;
                    ++count;
                    S = 1.0;
                    c = 0.0;
                    refused = 0;
                    left = __ballot(up == x);
                    continue;
                }
                refused |= 1ull << x;
                if (draft) {
                    c += S;
                    if (left) { sum = true; break; }        // (after the last child nobody asks for S)
                } else {
                    S = __builtin_fmax(S - r, 0.0);
                }
            }
            if (lane == 0) { at_node = node; at_c = c; at_refused = refused; need_sum = sum; }
        }
        __syncthreads();
        if (!need_sum) break;
        const Residual res{target + (size_t)at_node * a.stride, draft + (size_t)at_node * a.stride, at_c, -1, V};
        double mine = 0.0;
        for (int i = wv; i < a.chunks; i += VF_WAVES) mine += res.chunk_sum(i);
        if (lane == 0) wave_part[wv] = mine;
        __syncthreads();
        if (wv == 0) {
            S = 0.0;
#pragma unroll
            for (int w = 0; w < VF_WAVES; ++w) S += wave_part[w];
        }
    }
    if (counts && lane == 0) a.n_path[b] = count;

    // ---- the next token ----------------------------------------------------------------
    const bool is_refused = !draft && ((at_refused >> lane) & 1ull);
    Residual res{target + (size_t)at_node * a.stride, at_c != 0.0 ? draft + (size_t)at_node * a.stride : nullptr, at_c,
                 is_refused ? token : -1, V};
    double *sums = a.sums + (size_t)b * a.chunks;
    for (int i = share * VF_WAVES + wv; i < a.chunks; i += a.S * VF_WAVES) {
        const double s = res.chunk_sum(i);
        if (lane == 0) put(sums + i, s);
    }
    __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wave's sums have reached memory
    __syncthreads();
    if (a.S > 1) {
        if (threadIdx.x == 0) {
            // a byte of a status word per sequence
            int32_t *word = a.status + VF_FIRST_TICKET + b / 4;
            const int shift = 8 * (b & 3);
            const uint32_t old = (uint32_t)__hip_atomic_fetch_add(word, 1 << shift, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            is_last = (int)((old >> shift) & 0xFFu) == a.S - 1;
            if (is_last) __hip_atomic_fetch_add(word, -(a.S << shift), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!is_last) return;
    }
    __asm__ volatile("" ::: "memory");
    int token_out = draw_token(res, sums, a.chunks, us);     // (every wave the same)
    if (token_out < 0) {                                     // nothing left: p itself
        __syncthreads();
        res.q = nullptr;
        res.c = 0.0;
        res.refused = -1;
        for (int i = wv; i < a.chunks; i += VF_WAVES) {
            const double s = res.chunk_sum(i);
            if (lane == 0) put(sums + i, s);
        }
        __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        token_out = draw_token(res, sums, a.chunks, us);
        if (token_out < 0 && threadIdx.x == 0) atomicAdd(&a.status[NGC_STATUS_BAD_TREE], 1);
    }
    if (threadIdx.x == 0) a.next[b] = token_out;
    __syncthreads();
    for (int i = threadIdx.x; i < a.chunks; i += VF_THREADS) put(sums + i, 0.0);    // as it was found, in any workspace
}

}  // namespace ngc

// ============================================================ host side ====

using namespace ngc;

extern "C" size_t ngc_verify_workspace_bytes(int32_t B, int32_t V)
{
    if (B <= 0 || V <= 0) return 0;
    return STATUS_BYTES + (size_t)B * ((V + VF_CHUNK - 1) / VF_CHUNK) * sizeof(double);
}

extern "C" int ngc_tree_verify(const float *target, const float *draft, int64_t prob_stride, const int32_t *token,
                               const int32_t *parent, const int32_t *n_draft, int32_t B, int32_t W, int32_t V,
                               const float *u_accept, const float *u_sample, int32_t *path_out, int32_t *n_path_out,
                               int32_t *next_out, void *ws, size_t ws_bytes, void *stream)
{
    if (!target || !token || !parent || !u_accept || !u_sample || !path_out || !n_path_out || !next_out || !ws) return NGC_EINVAL;
    if (!aligned16(ws) || ((reinterpret_cast<uintptr_t>(target) | reinterpret_cast<uintptr_t>(draft)) & 3u)) return NGC_EINVAL;
    if (B <= 0 || W <= 0 || V <= 0 || prob_stride < V) return NGC_EINVAL;
    if (W > 64 || V > 0x7FFFFFFF - 2 * VF_CHUNK) return NGC_EUNSUPPORTED;
    if (ws_bytes < ngc_verify_workspace_bytes(B, V)) return NGC_ENOSPC;
    VerifyArgs a;
    a.target = target; a.draft = draft;
    a.token = token; a.parent = parent; a.n_draft = n_draft;
    a.u_accept = u_accept; a.u_sample = u_sample;
    a.path = path_out; a.n_path = n_path_out; a.next = next_out;
    a.status = reinterpret_cast<int32_t *>(ws);
    a.sums = reinterpret_cast<double *>(reinterpret_cast<unsigned char *>(ws) + STATUS_BYTES);
    a.stride = prob_stride;
    a.W = W; a.V = V;
    a.chunks = (V + VF_CHUNK - 1) / VF_CHUNK;
    int S = 512 / B;
    const int most = (a.chunks + VF_WAVES - 1) / VF_WAVES;
    S = S < most ? S : most;
    S = S < 64 ? S : 64;
    a.S = B > VF_TICKETS || S < 1 ? 1 : S;
    return launch(reinterpret_cast<const void *>(&verify_kernel), dim3(B, a.S), dim3(VF_THREADS), 0, (hipStream_t)stream, a);
}
