// Rotary positions for gfx950 and their C ABI entry point
// (include/sangam_rope.h).
//
// Every element is read once and written once, and a pair needs one sine and
// one cosine, the same for all heads of a row: the kernel is bound by HBM as
// long as those are computed once per row and not per head (some 40 instructions
// each, for a thread's own 8 pairs as many as the memory leaves time for). A
// work-group holds some rows and some heads: it computes the rows' angles into
// LDS (64-bit product, turns reduced to an eighth there, then fp32), and its
// threads rotate units of 16 bytes on either side of a pair (halves) or of
// 16 bytes of pairs (interleaved).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "../../include/sangam_rope.h"
#include "entry.h"
#include "rope_format.h"

namespace sangam {
void set_error(const std::string& msg);
void clear_error();
const RopePlanHeader* check_rope_plan(const void* plan);
}  // namespace sangam

using namespace sangam;

namespace {

struct RopeTensor {
    const void* in;
    void* out;
    int64_t in_row, in_head, out_row, out_head;
};

struct RopeArgs {
    RopeTensor t[2];  // q, k
    const double* turns;
    const int32_t* positions;
    int64_t rows;
    int32_t heads_q;
    int32_t heads;      // of q and k
    int32_t rot;
    int32_t head_dim;
    int32_t units;      // of a head: rotating ones, then ones to copy
    int32_t copy;       // dims of a head to copy
    int32_t in_place;   // whether q or k is rotated in place
    int32_t rows_each;  // rows of a work-group
    int32_t heads_each; // heads of a work-group
    float size_cos;     // factors on cos and sin
    float size_sin;
};

constexpr int kThreads = 256;
// Units that a thread loads together: 4099 rows of 40 heads of 64, fp32, with one
// 15.4 us, with two 14.9, with four 14.4 (5.8 TB/s); 15,627 of 64 heads of 128 97.1,
// 95.9, 95.1.
constexpr int kUnits = 4;
constexpr int kGroups = 8 * 256;  // work-groups that a launch has if it can

// Output bytes from which the stores are nontemporal. Measured with plain ->
// nontemporal stores, 64 heads of 128 dims: 33 MB 11.5 -> 12.1 us, 66 MB 28.5 ->
// 21.6, 131 MB 51.8 -> 50.3, 256 MB 98.3 -> 95.1, 983 MB 365 -> 360. (What is
// smaller stays in the cache for the attention that reads it next.)
constexpr int64_t kStreamBytes = int64_t(48) << 20;

// cos and sin of a number of turns given in 64 bits
__device__ __forceinline__ float2 cos_sin(double turns) {
    const double quarter = __builtin_rint(4.0 * turns);
    const float r = float(__builtin_fma(-0.25, quarter, turns));  // |r| <= 1/8
    float s, c;
    sincospif(2.0f * r, &s, &c);
    // quarters mod 4: 4 turns mod 4 is exact in 64 bits, and at most 2^33 here
    const int q = int(int64_t(quarter)) & 3;
    const float a = (q & 1) ? s : c, b = (q & 1) ? c : s;
    return float2{(q == 1 || q == 2) ? -a : a, q >= 2 ? -b : b};
}

// A pair turned by (cos, sin). Which product is fused is written out: every
// variant of the kernel gives the same bits.
__device__ __forceinline__ float turned0(float x0, float x1, float2 k) { return __builtin_fmaf(x0, k.x, -(x1 * k.y)); }
__device__ __forceinline__ float turned1(float x0, float x1, float2 k) { return __builtin_fmaf(x1, k.x, x0 * k.y); }
// (fp16: as a number of 32 bits first; a product and sum that end in 16 at once
// round once, and the compiler takes them in some places)
template <typename T>
__device__ __forceinline__ T rounded(float y) {
    if constexpr (sizeof(T) == 2 && !__is_same(T, __bf16)) asm("" : "+v"(y));
    return T(y);
}

template <bool STREAM, typename Access, typename V>
__device__ __forceinline__ void put(void* p, V v) {
    if (STREAM) __builtin_nontemporal_store(v, static_cast<V*>(p));
    else *static_cast<Access*>(p) = v;
}

// T: element; V: elements of a vector access
// EDGES: where a stride, an address or a number of pairs or of dims to copy does
// not allow whole, aligned vectors. Accesses are aligned to elements, and the last
// vector of the pairs, or of the dims to copy, moves back to end where they do:
// some outputs are computed and written twice, to the same bits. In place, where
// what it reads of its neighbour may be rotated already, it writes its own
// elements only. 4748 rows of 28 + 4 heads of 128 dims, 126 of them rotated, fp16:
// one element at a time 48.5 us, so 22.9, in place 38.9 and 22.8; 15,000 of 32 + 8 heads
// of 64, 18 rotated, bf16: 118.6 and 47.0, in place 34.0 and 29.8. (Twice what the
// bytes take: most vectors cross a line of 128 bytes, dims that only pass are
// units of their own, and the stores are plain ones at every size.)
template <typename T, int V, bool INTERLEAVED, bool STREAM, bool EDGES>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
    typedef T Vec __attribute__((ext_vector_type(V)));
    typedef Vec Access __attribute__((aligned(EDGES ? sizeof(T) : sizeof(Vec))));
    constexpr bool ONE = INTERLEAVED && V > 1;  // a unit is one vector of whole pairs, else the two sides of V pairs
    extern __shared__ float2 angles[];          // [rows_each][rot / 2]
    const int half = a.rot / 2;
    const int64_t row0 = int64_t(blockIdx.x) * a.rows_each;
    const int nrows = int(a.rows - row0 < a.rows_each ? a.rows - row0 : a.rows_each);
    const int head0 = int(blockIdx.y) * a.heads_each;
    const int nheads = min(a.heads_each, a.heads - head0);
    const int side = INTERLEAVED ? a.rot / (ONE ? 1 : 2) : half;  // elements that units of V cover
    const int rotating = EDGES ? (side + V - 1) / V : side / V;
    const int total = nrows * nheads * a.units;

    // A thread's next units, loaded together; those of the first round are on
    // their way while the angles are computed.
    struct Unit {
        Vec x, z;
        T* out;     // of its head; nullptr: no unit
        int first;  // dim of x
        int pairs;  // its first pair's entry in angles, -1: to copy, -2: to copy less than a vector
        int skip;   // elements of x that another unit writes
    } w[kUnits];
    auto load = [&](int u0) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            const int u = u0 + j * kThreads;
            w[j].out = nullptr;
            if (u >= total) continue;
            const int rh = u / a.units, c = u - rh * a.units;
            const int r = rh / nheads;
            int h = head0 + rh - r * nheads;
            const RopeTensor& t = a.t[h >= a.heads_q];
            if (h >= a.heads_q) h -= a.heads_q;
            const T* in = static_cast<const T*>(t.in) + (row0 + r) * t.in_row + h * t.in_head;
            w[j].out = static_cast<T*>(t.out) + (row0 + r) * t.out_row + h * t.out_head;
            const bool copy = c >= rotating;
            int at = copy ? (c - rotating) * V : c * V;
            w[j].skip = 0;
            if (EDGES) {
                const int whole = at;
                at = min(at, (copy ? a.copy : side) - V);
                if (a.in_place && !copy) w[j].skip = whole - at;
            }
            w[j].first = copy ? a.rot + at : ONE || !INTERLEAVED ? at : 2 * at;
            w[j].pairs = copy ? -1 : r * half + (ONE ? at / 2 : at);
            if (EDGES && copy && a.copy < V) {
                w[j].out += a.rot;
                w[j].pairs = -2;
                w[j].first = 0;
#pragma unroll
                for (int e = 0; e < V - 1; ++e)
                    if (e < a.copy) w[j].x[e] = in[a.rot + e];
                continue;
            }
            w[j].x = *(const Access*)(in + w[j].first);
            if (!ONE && !copy) w[j].z = *(const Access*)(in + w[j].first + (INTERLEAVED ? 1 : half));
        }
    };
    load(threadIdx.x);
    for (int k = threadIdx.x; k < nrows * half; k += kThreads) {
        const int r = k / half;
        const float2 cs = cos_sin(double(a.positions[row0 + r]) * a.turns[k - r * half]);
        angles[k] = float2{cs.x * a.size_cos, cs.y * a.size_sin};
    }
    __syncthreads();
    for (int u0 = threadIdx.x; u0 < total; u0 += kUnits * kThreads) {
        if (u0 != int(threadIdx.x)) load(u0);
#pragma unroll
        for (int j = 0; j < kUnits; ++j) {
            T* const out = w[j].out + w[j].first;
            if (!w[j].out) continue;
            if (EDGES && w[j].pairs == -2) {
#pragma unroll
                for (int e = 0; e < V - 1; ++e)
                    if (e < a.copy) out[e] = w[j].x[e];
                continue;
            }
            if (w[j].pairs < 0) {
                put<STREAM, Access>(out, w[j].x);
                continue;
            }
            const float2* cs = angles + w[j].pairs;
            Vec y, z;
            if constexpr (ONE) {
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float2 k = cs[e / 2];
                    const float x0 = float(w[j].x[e]), x1 = float(w[j].x[e + 1]);
                    y[e] = rounded<T>(turned0(x0, x1, k));
                    y[e + 1] = rounded<T>(turned1(x0, x1, k));
                }
                if (EDGES && w[j].skip > 0) {
#pragma unroll
                    for (int e = 1; e < V; ++e)
                        if (e >= w[j].skip) out[e] = y[e];
                    continue;
                }
                put<STREAM, Access>(out, y);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 k = cs[e];
                    const float x0 = float(w[j].x[e]), x1 = float(w[j].z[e]);
                    y[e] = rounded<T>(turned0(x0, x1, k));
                    z[e] = rounded<T>(turned1(x0, x1, k));
                }
                if (EDGES && w[j].skip > 0) {
#pragma unroll
                    for (int e = 1; e < V; ++e)
                        if (e >= w[j].skip) {
                            out[e] = y[e];
                            out[e + half] = z[e];
                        }
                    continue;
                }
                put<STREAM, Access>(out, y);
                put<STREAM, Access>(out + (INTERLEAVED ? 1 : half), z);
            }
        }
    }
}

enum class Access { kElements, kEdges, kVectors };

template <typename T, int V, bool INTERLEAVED>
const void* kernel_of(Access access, bool stream) {
    if (access == Access::kElements) return reinterpret_cast<const void*>(&rope_kernel<T, 1, INTERLEAVED, false, false>);
    if (access == Access::kEdges) return reinterpret_cast<const void*>(&rope_kernel<T, V, INTERLEAVED, false, true>);
    return stream ? reinterpret_cast<const void*>(&rope_kernel<T, V, INTERLEAVED, true, false>)
                  : reinterpret_cast<const void*>(&rope_kernel<T, V, INTERLEAVED, false, false>);
}
template <typename T, int V>
const void* kernel_of(Access access, bool interleaved, bool stream) {
    return interleaved ? kernel_of<T, V, true>(access, stream) : kernel_of<T, V, false>(access, stream);
}

sangam_status fail(sangam_status code, const std::string& msg) {
    set_error(msg);
    return code;
}

// Whether no two (row, head) of d elements overlap: the heads of a row side by
// side and rows apart from them, or the other way round.
bool apart(int64_t rows, int64_t row_stride, int64_t heads, int64_t head_stride, int64_t d) {
    if (row_stride < 0 || head_stride < 0) return false;
    const bool one_row = rows <= 1, one_head = heads <= 1;
    auto nested = [d](int64_t n, int64_t inner, bool one_inner, int64_t outer, bool one_outer) {
        if (!one_inner && inner < d) return false;
        const int64_t span = one_inner ? d : (n - 1) * inner + d;
        return one_outer || outer >= span;
    };
    return nested(heads, head_stride, one_head, row_stride, one_row) || nested(rows, row_stride, one_row, head_stride, one_head);
}

// A view [rows, heads, d] of elements.
struct View {
    uintptr_t at;
    int64_t row, head, heads;
};

// Whether two views may share an element: not where their spans, or, with the
// same step from row to row, their columns of a row are apart (views of one
// fused buffer).
bool may_overlap(const View& a, const View& b, int64_t rows, int64_t d, int64_t size) {
    const int64_t wa = (a.heads - 1) * a.head + d, wb = (b.heads - 1) * b.head + d;  // of a row
    const int64_t gap = (int64_t(b.at) - int64_t(a.at)) / size;
    if (gap >= (rows - 1) * a.row + wa || -gap >= (rows - 1) * b.row + wb) return false;
    if (a.row != b.row || a.row <= 0 || wa > a.row || wb > a.row) return true;
    const int64_t at = ((gap % a.row) + a.row) % a.row;  // b's first column, from a's
    return at < wa || at + wb > a.row;
}

constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxSpan = int64_t(1) << 48;  // of all rows, or of all heads, so that offsets fit 64 bits

sangam_status rotate(const void* plan_host, const void* plan_dev, const sangam_rope_tensor* q, const sangam_rope_tensor* k,
                     int32_t head_dim, int32_t dtype, const int32_t* positions_dev, int64_t rows, int32_t transpose, void* stream) {
    clear_error();
    const RopePlanHeader* h = check_rope_plan(plan_host);
    if (!h) return fail(SANGAM_ERR_PLAN, "plan_host is not a rotary plan of this library version");
    if (!q || rows < 0 || rows > INT32_MAX) return fail(SANGAM_ERR_INVALID_ARG, "q must not be NULL and rows must be 0 to 2^31 - 1");
    if (dtype != SANGAM_DTYPE_BF16 && dtype != SANGAM_DTYPE_FP16 && dtype != SANGAM_DTYPE_FP32)
        return fail(SANGAM_ERR_UNSUPPORTED, "dtype must be SANGAM_DTYPE_BF16, _FP16 or _FP32");
    if (head_dim < h->rot_dim || head_dim > kRopeMaxDim)
        return fail(SANGAM_ERR_INVALID_ARG, "head_dim must be the plan's rot_dim (" + std::to_string(h->rot_dim) + ") to 512");
    if (transpose != 0 && transpose != 1) return fail(SANGAM_ERR_INVALID_ARG, "transpose must be 0 or 1");
    const int64_t size = dtype == SANGAM_DTYPE_FP32 ? 4 : 2;
    const int V = int(16 / size);
    // vectors: whole ones on each side of the pairs, and every access aligned
    bool vectors = h->rot_dim % (h->interleaved ? V : 2 * V) == 0 && head_dim % V == 0;
    bool in_place = true, any_in_place = false;
    RopeArgs args{};
    int heads[2] = {0, 0};
    sangam_rope_tensor tensors[2] = {};
    for (int i = 0; i < 2; ++i) {
        if (!(i ? k : q)) continue;
        sangam_rope_tensor* t = &tensors[i];
        *t = i ? *k : *q;
        // the step of a single row or head leads nowhere
        if (rows <= 1) t->in_row_stride = t->out_row_stride = 0;
        if (t->heads == 1) t->in_head_stride = t->out_head_stride = 0;
        if (t->heads < 1 || t->heads > (1 << 16)) return fail(SANGAM_ERR_INVALID_ARG, "heads must be 1 to 2^16");
        heads[i] = t->heads;
        if (rows == 0) continue;
        if (!t->in || !t->out) return fail(SANGAM_ERR_INVALID_ARG, "the tensors must not be NULL");
        if (reinterpret_cast<uintptr_t>(t->in) % size || reinterpret_cast<uintptr_t>(t->out) % size)
            return fail(SANGAM_ERR_ALIGN, "the tensors must be aligned to their elements");
        if (t->in_row_stride < 0 || t->in_head_stride < 0 || t->in_row_stride > kMaxStride || t->in_head_stride > kMaxStride ||
            t->out_row_stride > kMaxStride || t->out_head_stride > kMaxStride)
            return fail(SANGAM_ERR_INVALID_ARG, "strides must be 0 to 2^40");
        if (std::max(t->in_row_stride, t->out_row_stride) > kMaxSpan / rows || std::max(t->in_head_stride, t->out_head_stride) > kMaxSpan / t->heads)
            return fail(SANGAM_ERR_INVALID_ARG, "rows times their stride and heads times theirs must be 0 to 2^48");
        if (!apart(rows, t->out_row_stride, t->heads, t->out_head_stride, head_dim))
            return fail(SANGAM_ERR_INVALID_ARG, "rows and heads of the output overlap");
        if (t->in == t->out && (t->in_row_stride != t->out_row_stride || t->in_head_stride != t->out_head_stride))
            return fail(SANGAM_ERR_INVALID_ARG, "a tensor rotated in place must keep its strides");
        for (int64_t stride : {t->in_row_stride, t->in_head_stride, t->out_row_stride, t->out_head_stride}) vectors = vectors && stride % V == 0;
        vectors = vectors && reinterpret_cast<uintptr_t>(t->in) % 16 == 0 && reinterpret_cast<uintptr_t>(t->out) % 16 == 0;
        in_place = in_place && t->in == t->out;
        any_in_place = any_in_place || t->in == t->out;
        args.t[i] = RopeTensor{t->in, t->out, t->in_row_stride, t->in_head_stride, t->out_row_stride, t->out_head_stride};
    }
    if (rows == 0) return SANGAM_OK;
    View views[4];  // inputs, outputs
    for (int i = 0; i < 2; ++i) {
        const RopeTensor& t = args.t[i];
        views[i] = View{reinterpret_cast<uintptr_t>(t.in), t.in_row, t.in_head, heads[i]};
        views[2 + i] = View{reinterpret_cast<uintptr_t>(t.out), t.out_row, t.out_head, heads[i]};
    }
    for (int o = 0; o < (k ? 2 : 1); ++o)
        for (int i = 0; i < (k ? 2 : 1); ++i)
            if (!(o == i && args.t[o].in == args.t[o].out) && may_overlap(views[i], views[2 + o], rows, head_dim, size))
                return fail(SANGAM_ERR_INVALID_ARG, std::string(o ? "k's" : "q's") + " output overlaps " + (i ? "k" : "q") + " without being it");
    if (k && may_overlap(views[2], views[3], rows, head_dim, size)) return fail(SANGAM_ERR_INVALID_ARG, "the outputs overlap");
    if (!plan_dev || !positions_dev) return fail(SANGAM_ERR_INVALID_ARG, "plan_dev and positions_dev must not be NULL");
    if (reinterpret_cast<uintptr_t>(plan_dev) & 15u || reinterpret_cast<uintptr_t>(positions_dev) & 3u)
        return fail(SANGAM_ERR_ALIGN, "plan_dev must be 16-byte and positions_dev 4-byte aligned");
    // edges: a vector of pairs at least
    const bool short_side = h->rot_dim < (h->interleaved ? V : 2 * V);
    const Access access = vectors ? Access::kVectors : short_side ? Access::kElements : Access::kEdges;
    const int v = access == Access::kElements ? 1 : V;
    args.turns = reinterpret_cast<const double*>(static_cast<const uint8_t*>(plan_dev) + h->off_turns);
    args.heads_q = heads[0];
    args.heads = heads[0] + heads[1];
    args.rot = h->rot_dim;
    args.head_dim = head_dim;
    args.copy = in_place ? 0 : head_dim - h->rot_dim;
    args.in_place = any_in_place;
    const int side = h->interleaved && v > 1 ? h->rot_dim : h->rot_dim / 2;
    args.units = (side + v - 1) / v + (args.copy + v - 1) / v;
    args.size_cos = h->magnitude;
    args.size_sin = transpose ? -h->magnitude : h->magnitude;
    // A work-group: up to four rows of all heads; fewer rows, and then fewer
    // heads while each thread has more than one unit, where the launch has
    // under eight work-groups per CU (1536 rows of 32 heads, 768 -> 1536
    // work-groups, 8.2 -> 7.6 us; more rows each take the same time).
    args.rows_each = 4;
    args.heads_each = args.heads;
    auto groups = [&] { return (rows + args.rows_each - 1) / args.rows_each * ((args.heads + args.heads_each - 1) / args.heads_each); };
    while (groups() < kGroups && args.rows_each > 1) args.rows_each /= 2;
    while (groups() < kGroups && int64_t(args.rows_each) * args.heads_each * args.units > kThreads && args.heads_each > 1)
        args.heads_each = (args.heads_each + 1) / 2;
    const bool nt = rows * args.heads * head_dim * size > kStreamBytes;
    const void* fn = dtype == SANGAM_DTYPE_FP32   ? kernel_of<float, 4>(access, h->interleaved, nt)
                     : dtype == SANGAM_DTYPE_FP16 ? kernel_of<_Float16, 8>(access, h->interleaved, nt)
                                                  : kernel_of<__bf16, 8>(access, h->interleaved, nt);
    void* kargs[] = {&args};
    const unsigned lds = unsigned(args.rows_each) * unsigned(h->rot_dim / 2) * unsigned(sizeof(float2));
    const unsigned splits = unsigned((args.heads + args.heads_each - 1) / args.heads_each);
    // a grid's threads are counted in 32 bits in each direction
    const int64_t step = ((int64_t(1) << 32) / kThreads - 1) * args.rows_each;  // rows of a launch
    const RopeTensor first[2] = {args.t[0], args.t[1]};
    for (int64_t row = 0; row < rows; row += step) {
        args.rows = std::min(step, rows - row);
        args.positions = positions_dev + row;
        for (int i = 0; i < 2; ++i) {
            args.t[i].in = static_cast<const uint8_t*>(first[i].in) + row * first[i].in_row * size;
            args.t[i].out = static_cast<uint8_t*>(first[i].out) + row * first[i].out_row * size;
        }
        const hipError_t e = hipLaunchKernel(fn, dim3(unsigned((args.rows + args.rows_each - 1) / args.rows_each), splits), dim3(kThreads),
                                             kargs, lds, static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return fail(SANGAM_ERR_HIP, std::string("rotary launch: ") + hipGetErrorString(e));
    }
    return SANGAM_OK;
}

}  // namespace

extern "C" sangam_status sangam_rope_rotate(const void* plan_host, const void* plan_dev, const sangam_rope_tensor* q,
                                            const sangam_rope_tensor* k, int32_t head_dim, int32_t dtype,
                                            const int32_t* positions_dev, int64_t rows, int32_t transpose, void* stream) {
    return entry([&] { return rotate(plan_host, plan_dev, q, k, head_dim, dtype, positions_dev, rows, transpose, stream); });
}
