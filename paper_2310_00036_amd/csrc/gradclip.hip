// The global norm over many gradient tensors and their clipped values. HBM-bound: every source is read once for the norm
// and once more for the values (from the caches where it fits them), every target written once. The tensors go by tables
// in the kernels' arguments, so that a call is two launches for up to kGcTable of them and copies nothing to the device.
// 36 tensors of 1.09 M float32 numbers in all: kernels of 5.0 and 7.0 us in the trace; 84 of 219 M, nearly all bf16, into float32:
// 370 us (381 on another card), 4.7 TB/s with the second reading.
#include <algorithm>

#include "common.h"
#include "gradclip.h"
#include "kernels.h"

namespace cb {

namespace {

constexpr int kGcTable = 96;       // tensors of a launch
constexpr int kGcSeg = 16384;       // elements a workgroup takes at a time
constexpr int kGcBlocks = 4096;    // workgroups of a launch, each with one partial sum (2048: 382 us for
                                   // the four wide blocks instead of 370)

struct GcEntry {
    const void* src;
    void* dst;
    int64_t n;
    int32_t type;                  // bit 0: src float32, bit 1: dst float32
};
struct GcTable {
    GcEntry e[kGcTable];
    int32_t first[kGcTable];       // an entry's first segment in the launch; behind the last, more than there are
    int n, segs;
};
static_assert(kGcTable <= 128 && sizeof(GcTable) <= 3584, "two entries a lane, and a kernel's arguments");

// 16 bytes at any alignment of an element: global memory takes them so.
typedef uint32_t gc_u32x4 __attribute__((ext_vector_type(4), aligned(2)));

// f(entry, first element, elements) for this workgroup's segments, which are neighbours: the tensor of the first one is
// looked up, the others follow from it. `back` takes the workgroups and their segments from the end.
template <class F>
CB_DEV void gc_segments(const GcTable& t, bool back, F&& f) {
    const int b = back ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    const int s0 = int(int64_t(t.segs) * b / gridDim.x), s1 = int(int64_t(t.segs) * (b + 1) / gridDim.x);
    if (s0 >= s1) return;
    // the last entry that starts at or before the first segment: lanes compare, two entries each
    const int s = back ? s1 - 1 : s0, lane = threadIdx.x & 63;
    const int more = min(lane + 64, kGcTable - 1);
    int at = __popcll(__ballot(t.first[lane] <= s)) + __popcll(__ballot(more == lane + 64 && t.first[more] <= s)) - 1;
    for (int i = 0; i < s1 - s0; ++i) {
        const int s = back ? s1 - 1 - i : s0 + i;
        if (back) { if (s < t.first[at]) --at; }
        else if (at + 1 < t.n && s >= t.first[at + 1]) ++at;
        const GcEntry& e = t.e[at];
        const int64_t el = int64_t(s - t.first[at]) * kGcSeg;
        f(e, el, int(min(int64_t(kGcSeg), e.n - el)));
    }
}

// Eight elements of a source, `left` of which exist: one or two 16-byte words, and as floats.
struct GcRaw { gc_u32x4 a, b; };
template <bool F32>
CB_DEV GcRaw gc_raw(const GcEntry& e, int64_t i, int left) {
    GcRaw r;
    if constexpr (F32) {
        const float* p = static_cast<const float*>(e.src) + i;
        if (left >= 8) {
            r.a = *reinterpret_cast<const gc_u32x4*>(p);
            r.b = *reinterpret_cast<const gc_u32x4*>(p + 4);
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                r.a[u] = u < left ? __float_as_uint(p[u]) : 0u;
                r.b[u] = 4 + u < left ? __float_as_uint(p[4 + u]) : 0u;
            }
        }
    } else {
        const uint16_t* p = static_cast<const uint16_t*>(e.src) + i;
        if (left >= 8) r.a = *reinterpret_cast<const gc_u32x4*>(p);
        else
#pragma unroll
            for (int u = 0; u < 4; ++u)
                r.a[u] = (2 * u < left ? uint32_t(p[2 * u]) : 0u) | (2 * u + 1 < left ? uint32_t(p[2 * u + 1]) << 16 : 0u);
        r.b = r.a;
    }
    return r;
}
template <bool F32>
CB_DEV void gc_floats(const GcRaw& r, float* x) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if constexpr (F32) { x[u] = __uint_as_float(r.a[u]); x[4 + u] = __uint_as_float(r.b[u]); }
        else { x[2 * u] = bf_lo(r.a[u]); x[2 * u + 1] = bf_hi(r.a[u]); }
    }
}

// f(offset, elements left, eight floats) over a segment, 128 bytes of a thread on their way at once (64: 384 us for the
// four wide blocks instead of 370).
template <bool F32, class F>
CB_DEV void gc_pieces(const GcEntry& e, int64_t at, int n, F&& f) {
    constexpr int ST = 8 * 256, NP = F32 ? 4 : 8;
    for (int i0 = 8 * int(threadIdx.x); i0 < n; i0 += NP * ST) {
        GcRaw r[NP];
#pragma unroll
        for (int u = 0; u < NP; ++u) r[u] = gc_raw<F32>(e, at + i0 + u * ST, n - i0 - u * ST);
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            if (i0 + u * ST >= n) break;
            float x[8];
            gc_floats<F32>(r[u], x);
            f(at + i0 + u * ST, n - i0 - u * ST, x);
        }
    }
}

// `bits`: what came from bf16 goes there as it came (a conversion would make signalling NaN quiet).
CB_DEV void gc_store8(const GcEntry& e, int64_t i, int left, const float* x, bool bits) {
    if (e.type & 2) {
        float* p = static_cast<float*>(e.dst) + i;
        if (left >= 8) {
            gc_u32x4 a, b;
#pragma unroll
            for (int u = 0; u < 4; ++u) { a[u] = __float_as_uint(x[u]); b[u] = __float_as_uint(x[4 + u]); }
            *reinterpret_cast<gc_u32x4*>(p) = a;
            *reinterpret_cast<gc_u32x4*>(p + 4) = b;
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (u < left) p[u] = x[u];
        }
    } else {
        uint16_t* p = static_cast<uint16_t*>(e.dst) + i;
        if (left >= 8) {
            gc_u32x4 a;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                a[u] = bits ? __float_as_uint(x[2 * u]) >> 16 | (__float_as_uint(x[2 * u + 1]) & 0xffff0000u)
                            : pack2bf(x[2 * u], x[2 * u + 1]);
            *reinterpret_cast<gc_u32x4*>(p) = a;
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (u < left) p[u] = bits ? uint16_t(__float_as_uint(x[u]) >> 16) : f2bf(x[u]);
        }
    }
}

// Squares are summed in 64 bits: a float32 number's square fits them, whatever its size.
__global__ __launch_bounds__(256) void gc_norm_kernel(GcTable t, double* part) {
    __shared__ double sh[256];
    double s = 0.0;
    gc_segments(t, false, [&](const GcEntry& e, int64_t at, int n) {
        auto add = [&](int64_t, int, const float* x) {
#pragma unroll
            for (int u = 0; u < 8; ++u) s += double(x[u]) * x[u];
        };
        e.type & 1 ? gc_pieces<true>(e, at, n, add) : gc_pieces<false>(e, at, n, add);
    });
    const double tot = block_sum<256>(s, sh);
    if (threadIdx.x == 0) part[blockIdx.x] = tot;
}

CB_DEV double gc_total(const double* part, int nparts, double* sh) {
    double s = 0.0;
    for (int i = threadIdx.x; i < nparts; i += 256) s += part[i];
    return block_sum<256>(s, sh);
}

// Many partial sums to one, where they are of several launches.
__global__ __launch_bounds__(256) void gc_sum_kernel(const double* part, int nparts, double* total) {
    __shared__ double sh[256];
    const double s = gc_total(part, nparts, sh);
    if (threadIdx.x == 0) *total = s;
}

__global__ __launch_bounds__(256) void gc_scale_kernel(GcTable t, const double* part, int nparts, float max_norm, float* stats) {
    __shared__ double sh[256];
    const double norm = sqrt(gc_total(part, nparts, sh));
    if (stats && blockIdx.x == 0 && threadIdx.x == 0) {
        const float n = float(norm);
        stats[0] = n;
        stats[1] = isfinite(n) ? 0.f : 1.f;   // also where the norm is beyond float32
    }
    const bool clip = max_norm > 0.f && norm > double(max_norm);
    const float f = clip ? float(double(max_norm) / norm) : 1.f;
    // from the end: what the norm read last is still in the caches
    gc_segments(t, true, [&](const GcEntry& e, int64_t at, int n) {
        if (!e.dst || (!clip && e.dst == e.src)) return;
        auto put = [&](int64_t i, int left, float* x) {
            if (clip)
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] *= f;
            gc_store8(e, i, left, x, !clip && !(e.type & 1));
        };
        e.type & 1 ? gc_pieces<true>(e, at, n, put) : gc_pieces<false>(e, at, n, put);
    });
}

// Fills a table with tensors from i on; returns the next tensor. Empty ones are passed over.
int gc_fill(GcTable& t, const grad_tensor_t* g, int i, int n) {
    t.n = 0;
    int64_t segs = 0;
    for (; i < n && t.n < kGcTable; ++i) {
        if (g[i].count == 0) continue;
        const int64_t k = (g[i].count + kGcSeg - 1) / kGcSeg;
        if (t.n > 0 && segs + k > (int64_t(1) << 30)) break;
        t.first[t.n] = int32_t(segs);
        t.e[t.n++] = GcEntry{g[i].src, g[i].dst, g[i].count,
                             (g[i].src_prec == IMPALA_PREC_FP32 ? 1 : 0) | (g[i].dst_prec == IMPALA_PREC_FP32 ? 2 : 0)};
        segs += k;
    }
    t.segs = int(segs);
    for (int k = t.n; k < kGcTable; ++k) t.first[k] = INT32_MAX;
    return i;
}

int gc_blocks(const GcTable& t) { return std::min(t.segs, kGcBlocks); }

}  // namespace

size_t grad_clip_ws_bytes(const grad_tensor_t* g, int n) {
    GcTable t;
    int64_t parts = 1;
    for (int i = 0; i < n;) {
        i = gc_fill(t, g, i, n);
        parts += gc_blocks(t);
    }
    return size_t(parts) * sizeof(double);
}

hipError_t grad_clip_run(const grad_tensor_t* g, int n, float max_norm, float* stats, void* ws, hipStream_t s) {
    double* total = static_cast<double*>(ws);
    double* part = total + 1;
    ProfScope ps(s, [&] { return "grad_clip/" + std::to_string(n); });
    GcTable t;
    int nparts = 0, launches = 0;
    for (int i = 0; i < n;) {
        i = gc_fill(t, g, i, n);
        if (t.n == 0) break;
        hipLaunchKernelGGL(gc_norm_kernel, dim3(unsigned(gc_blocks(t))), dim3(256), 0, s, t, part + nparts);
        nparts += gc_blocks(t);
        ++launches;
    }
    if (launches != 1) {
        hipLaunchKernelGGL(gc_sum_kernel, dim3(1), dim3(256), 0, s, part, nparts, total);
        part = total;
        nparts = 1;
    }
    int done = 0;
    for (int i = 0; i < n || done == 0; ++done) {
        i = gc_fill(t, g, i, n);
        if (t.n == 0 && done > 0) break;
        hipLaunchKernelGGL(gc_scale_kernel, dim3(unsigned(std::max(1, gc_blocks(t)))), dim3(256), 0, s, t, part, nparts,
                           max_norm, done == 0 ? stats : nullptr);
    }
    return hipGetLastError();
}

}  // namespace cb
