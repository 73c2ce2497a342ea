// libsbc: host side of the operators in include/sbc.h that work without a context (microscaled 4-bit
// matrices, top logits, distillation).  Each call checks its arguments, chooses among the kernels and
// enqueues them on the caller's stream; none allocates, copies or waits.
#include "../../include/sbc.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "sbc_mxfp_kernels.hpp"
#include "sbc_logits_kernels.hpp"

using namespace sbc;

namespace {

struct DeviceScope {
    int prev = -1;
    bool changed = false;
    explicit DeviceScope(int dev) {
        if (hipGetDevice(&prev) == hipSuccess && prev != dev) changed = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceScope() { if (changed) (void)hipSetDevice(prev); }
};

int device_status(int device) {
    int n = 0;
    if (device < 0) return SBC_EINVAL;
    if (hipGetDeviceCount(&n) != hipSuccess) { (void)hipGetLastError(); return SBC_EHIP; }
    return device < n ? SBC_OK : SBC_EINVAL;
}

constexpr int64_t kMostDim = (int64_t)1 << 31;          // rows and columns stay below
constexpr int64_t kMostGroups = (int64_t)1 << 22;       // workgroups of a launch (the runtime takes 2^32 work items)

size_t size_of(int type) { return type == SBC_F32 ? 4 : type == SBC_BF16 || type == SBC_F16 ? 2 : 0; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool dim_ok(int64_t n) { return n >= 1 && n < kMostDim; }
// a dense matrix of `rows` rows, ld values apart
bool dense_ok(const void* x, int type, int64_t cols, int64_t ld) { return x && size_of(type) && aligned(x, size_of(type)) && ld >= cols && ld < ((int64_t)1 << 40); }
bool held_ok(const void* q) { return q && aligned(q, 16); }

// The memory of an argument: `rows` runs of `run` bytes, `ld` bytes from one to the next.  None for a null pointer.
struct Span {
    uintptr_t from = 0, end = 0;
    uint64_t rows = 0, run = 0, ld = 0;
    Span(const void* p, uint64_t rows_, uint64_t run_, uint64_t ld_) {
        if (!p || !rows_ || !run_) return;
        from = reinterpret_cast<uintptr_t>(p);
        rows = rows_;
        run = run_;
        ld = ld_;
        uint64_t past;                                         // (beyond all addresses where the product is)
        if (__builtin_mul_overflow(rows - 1, ld, &past) || __builtin_add_overflow(past, run, &past) || __builtin_add_overflow(past, from, &past)) past = UINT64_MAX;
        end = past;
    }
    Span(const void* p, uint64_t bytes) : Span(p, 1, bytes, bytes) {}
};
Span matrix_span(const void* p, int type, int64_t rows, int64_t cols, int64_t ld) {
    const uint64_t size = size_of(type);
    return {p, (uint64_t)rows, (uint64_t)cols * size, (uint64_t)ld * size};
}

// Whether two arguments share no byte.  Rows the same distance apart may lie beside each other in one buffer; of other
// matrices that lie among each other it is not said.
bool apart(const Span& a, const Span& b) {
    if (!a.rows || !b.rows || a.end <= b.from || b.end <= a.from) return true;
    if (a.rows == 1 && b.rows == 1) return false;
    const uint64_t ld = a.rows > 1 ? a.ld : b.ld;
    if (b.rows > 1 && b.ld != ld) return false;
    const uint64_t behind = b.from >= a.from ? (b.from - a.from) % ld : ld - 1 - (a.from - b.from - 1) % ld;      // of b's runs' starts behind a's
    return a.run <= behind && behind + b.run <= ld;
}

// Whether what a call writes is apart from itself and from what it reads.
bool apart(std::initializer_list<Span> written, std::initializer_list<Span> read) {
    for (const Span* w = written.begin(); w != written.end(); ++w) {
        for (const Span* other = written.begin(); other != w; ++other)
            if (!apart(*w, *other)) return false;
        for (const Span& r : read)
            if (!apart(*w, r)) return false;
    }
    return true;
}
Span held_span(const void* q, int64_t rows, int64_t cols) { return {q, (uint64_t)(mx_panels(rows) * mx_steps(cols)) * (kMxPanelBytes + kMxScaleBytes)}; }

MxPtr container(const void* q, int64_t rows, int64_t cols) {
    uint8_t* const p = static_cast<uint8_t*>(const_cast<void*>(q));
    return {p, p + mx_panels(rows) * mx_steps(cols) * kMxPanelBytes};
}

int launched() { return hipGetLastError() == hipSuccess ? SBC_OK : SBC_EHIP; }

// f(T()) with the C++ type of a value type
template <typename F> int by_type(int type, F f) {
    switch (type) {
        case SBC_F32: return f(float());
        case SBC_BF16: return f(__bf16());
        case SBC_F16: return f(_Float16());
        default: return SBC_EINVAL;
    }
}

// f(first row, rows) for slices of the rows whose workgroups one launch can have
template <typename F> void by_rows_of(int64_t rows, int64_t groups_per_row, F f) {
    const int64_t most = std::max<int64_t>(1, kMostGroups / groups_per_row);
    for (int64_t r = 0; r < rows; r += most) f(r, std::min(most, rows - r));
}

template <typename T>
void launch_quantize(hipStream_t stream, const void* x, int64_t rows, int64_t cols, int64_t ld, void* by_rows, void* by_cols) {
    const MxPtr r = container(by_rows, rows, cols), c = container(by_cols, cols, rows);
    const T* const in = static_cast<const T*>(x);
    const dim3 block(kMxQuantThreads);
    if (!by_cols) {
        const uint32_t steps = (uint32_t)mx_steps(cols);
        hipLaunchKernelGGL((k_mxfp_quantize_rows<T>), dim3((uint32_t)mx_panels(rows) * steps), block, 0, stream, in, ld, rows, cols, steps, r);
        return;
    }
    const int64_t wide = by_rows || sizeof(T) == 2 ? 128 : 64, high = by_rows ? kMxPanel : 128;
    const uint32_t tr = (uint32_t)((rows + high - 1) / high), tc = (uint32_t)((cols + wide - 1) / wide);
    if (by_rows) hipLaunchKernelGGL((k_mxfp_quantize<T>), dim3(tr * tc), block, 0, stream, in, ld, rows, cols, tc, r, c);
    else hipLaunchKernelGGL((k_mxfp_quantize_cols<T>), dim3(tr * tc), block, 0, stream, in, ld, rows, cols, tc, c);
}

template <typename T, int PM, int PN, int WM, int WN, int kStages, int kSplit>
void launch_tiles(hipStream_t stream, MxPtr a, MxPtr b, int64_t M, int64_t N, int64_t K, T* c, int64_t ldc) {
    const uint32_t tm = (uint32_t)((mx_panels(M) + PM - 1) / PM), tn = (uint32_t)((mx_panels(N) + PN - 1) / PN);
    hipLaunchKernelGGL((k_mxfp_matmul<T, PM, PN, WM, WN, kStages, kSplit>), dim3(tm * tn), dim3(64 * WM * WN * kSplit), 0, stream, a, b, M, N, (uint32_t)mx_steps(K), tm, tn, c, ldc);
}

// 128 x 128 outputs to a workgroup, three workgroups to a compute unit.  Where no compute unit has a second one anyway,
// it is the waits of a step that count, and twice the wavefronts share the steps (us, one part / two: 2048 x 2048 x 8192 22.6 /
// 20.6, 256 x 8192 x 8192 20.7 / 17.5, 699 x 1500 x 10000 25.4 / 21.1; but 2799 x 1500 x 10000, 264 workgroups, 38 / 45).
template <typename T>
void launch_matmul(hipStream_t stream, MxPtr a, MxPtr b, int64_t M, int64_t N, int64_t K, T* c, int64_t ldc) {
    if (((M + 127) / 128) * ((N + 127) / 128) <= 256) launch_tiles<T, 2, 2, 2, 2, 3, 2>(stream, a, b, M, N, K, c, ldc);
    else launch_tiles<T, 2, 2, 2, 2, 3, 1>(stream, a, b, M, N, K, c, ldc);
}

// Few rows: how many tiles of 16 rows of B a workgroup takes.  A compute unit reads a tile's step in about 51 ns where all
// of them read, and rounds a block of A in 0.46 ns of its 256 threads' time; the workgroups come in rounds of 256.
int few_tiles(int64_t N, int64_t steps, int64_t blocks) {
    const int64_t tiles = (N + 15) / 16;
    int best = 1;
    double least = 0.0;
    for (int tw = 1; tw <= 4; tw *= 2) {
        const double t = (double)(((tiles + tw - 1) / tw + 255) / 256) * ((double)(tw * steps) * 51.0 + (double)blocks * 0.46);
        if (tw == 1 || t < least) { best = tw; least = t; }
    }
    return best;
}

// Whether the workgroups round few rows of A for themselves: 36 KB of LDS at most, and, but for so few values that it hardly
// matters, not by so many workgroups that it costs more than a launch that rounds them once (us, by themselves / beforehand:
// 1 x 10000 x 1500 7.6 / 13.1, 8 x 16384 x 8192 18.0 / 20.3, 4 x 100000 x 1500 19.9 / 21.6; but 16 x 50000 x 4096 48 / 31, 16 x 32768 x
// 4096 25 / 21).
constexpr int64_t kFewMost = 65536, kFewAlways = 16384, kFewAll = (int64_t)1 << 24, kFewGroups = 1024;

int64_t few_values(int64_t M, int64_t K) { return M <= 16 ? M * mx_steps(K) * kMxStep : kFewMost + 1; }

bool few_fused(int64_t M, int64_t N, int64_t K) {
    const int64_t values = few_values(M, K);
    if (values <= kFewAlways || values > kFewMost) return values <= kFewMost;
    const int64_t per = 16 * few_tiles(N, mx_steps(K), values / 32), groups = (N + per - 1) / per;
    return groups <= kFewGroups && groups * values <= kFewAll;
}

template <typename T, int TW, int CT, bool kFused, int kWaves = 4>
void launch_few(hipStream_t stream, const T* x, int64_t ldx, MxPtr a, int64_t M, int64_t K, MxPtr b, int64_t N, T* c, int64_t ldc) {
    const int64_t steps = mx_steps(K), groups = ((N + 15) / 16 + TW - 1) / TW;
    const size_t rows = kFused ? (size_t)(steps * 4 * M) * 17 : 0, sums = (size_t)TW * CT * kWaves * 64 * 16;
    hipLaunchKernelGGL((k_mxfp_few<T, TW, CT, kFused, kWaves>), dim3((uint32_t)groups, (uint32_t)(kFused ? 1 : mx_panels(M))), dim3(64 * kWaves), (uint32_t)((std::max(rows, sums) + 15) / 16 * 16), stream, x, ldx, a, M, K, b, N,
                       (uint32_t)steps, c, ldc);
}

template <typename T, int CT, bool kFused>
void launch_few_tiles(hipStream_t stream, const T* x, int64_t ldx, MxPtr a, int64_t M, int64_t K, MxPtr b, int64_t N, T* c, int64_t ldc) {
    const int64_t steps = mx_steps(K);
    switch (few_tiles(N, steps, kFused ? steps * 4 * M : 0)) {
        case 1: launch_few<T, 1, CT, kFused>(stream, x, ldx, a, M, K, b, N, c, ldc); break;
        case 2: launch_few<T, 2, CT, kFused>(stream, x, ldx, a, M, K, b, N, c, ldc); break;
        default: launch_few<T, 4, CT, kFused, 8>(stream, x, ldx, a, M, K, b, N, c, ldc);      // (a workgroup to a compute unit: 8 x 16384 x 8192 20.9 us with four wavefronts, 17.5 with eight)
    }
}

// Small products have k_mxfp_few's shapes for every panel of A: nothing goes through LDS, and there are more workgroups
// (us with the rounding of A, 128 x 128 outputs / this: 64 x 1500 x 10000 23.7 / 18.8, 32 x 12000 x 4096 15.1 / 12.8, 128 x 4096 x 4096
// 14.6 / 12.8, 500 x 1500 x 10000, 192 panels, 28.6 / 27.0; but 128 x 8192 x 8192, 256 panels, 21.7 / 24.0, 300 x 4000 x 1000, 315,
// 12.1 / 13.9).
constexpr int64_t kFewPanels = 200;

template <typename T>
void launch_product(hipStream_t stream, MxPtr a, MxPtr b, int64_t M, int64_t N, int64_t K, T* c, int64_t ldc) {
    if (M <= 16) launch_few_tiles<T, 1, false>(stream, nullptr, 0, a, M, K, b, N, c, ldc);
    else if (mx_panels(M) * mx_panels(N) > kFewPanels) launch_matmul<T>(stream, a, b, M, N, K, c, ldc);
    else if (M <= 32) launch_few<T, 1, 2, false>(stream, nullptr, 0, a, M, K, b, N, c, ldc);
    else if (M <= 128) launch_few<T, 1, 4, false>(stream, nullptr, 0, a, M, K, b, N, c, ldc);
    else launch_few<T, 4, 4, false>(stream, nullptr, 0, a, M, K, b, N, c, ldc);
}

bool tiles_fit(int64_t rows, int64_t cols) { return ((rows + 127) / 128) * ((cols + 127) / 128) <= kMostGroups; }

// (products of up to 16 rows have a workgroup for as few as 16 columns)
bool product_fits(int64_t M, int64_t N) { return tiles_fit(M, N) && (M > 16 || N <= (int64_t)1 << 26); }

// How a row of `vocab` logits is dealt out: parts of `vecs` vectors of eight.
struct RowPlan { uint32_t parts, vecs; };

// A workgroup per row where that fills the chip or the row is short: the second launch and the join cost 4 to 10 us, the more
// the longer the lists (us, one / parts: one row of 20000, k = 64 12.6 / 16.5, of 50021 18.5 / 14.4, of 131072 31 / 14; of 50021
// with k = 238 24.5 / 29.4; 100 rows of 50021 20.7 / 23.6, of 131072 32 / 29).  Else as many parts as give about kTopGroups
// workgroups, of two vectors a thread at least, and so few that the join holds all of their keys.
constexpr int64_t kTopGroups = 512;
constexpr int64_t kTopShort = 4096;      // vectors
constexpr int64_t kTopShortListed = 16;  // ... and for each that is listed
constexpr int64_t kTopRowVecs = 96;      // vectors of a row for each row

RowPlan top_plan(int64_t rows, int64_t vocab, int k) {
    const int64_t vecs = (vocab + 14) / 8;                      // (wherever the row starts)
    const int64_t least = 2 * kTopThreads;
    int64_t parts = std::min<int64_t>({kTopGroups / rows, (vecs + least - 1) / least, (int64_t)(kJoinKeys / k)});
    if (parts < 3 || vecs <= kTopShort + kTopShortListed * k || vecs / rows < kTopRowVecs) parts = 1;
    const int64_t each = (vecs + parts - 1) / parts;
    return {(uint32_t)((vecs + each - 1) / each), (uint32_t)each};
}

// Short rows have two vectors for each of 256 threads and no more; many of them with short lists go one to a wavefront
// (6000 x 2025, k = 8 28 -> 17 us, 32 31 -> 22, 64 37 -> 35, but 250 87 -> 104; 1500 rows, k = 64 13 -> 18; 4096 x 50021 99 -> 131).
constexpr int64_t kTopManyRows = 2048;
constexpr int kTopManyListed = 64;

template <typename T, int n, int threads>
void launch_top(hipStream_t stream, int64_t groups, const T* x, int64_t ld, int64_t vocab, int k, const RowPlan& p, float inv_t, float c, const TopOut& out,
                unsigned long long* keys, ExpSum* sums) {
    hipLaunchKernelGGL((k_top<T, n, threads>), dim3((uint32_t)groups), dim3(threads), 0, stream, x, ld, (uint32_t)vocab, (uint32_t)k, p.parts, p.vecs, inv_t, c, out, keys, sums);
}

size_t top_room(int64_t rows, int64_t vocab, int k) {
    const RowPlan p = top_plan(rows, vocab, k);
    return p.parts == 1 ? 0 : (size_t)rows * p.parts * ((size_t)k * sizeof(unsigned long long) + sizeof(ExpSum));
}

// A workgroup takes a row (parts = 1): at once if it has the registers for it, else in passes where there are rows
// enough or the row is not so long that it takes longer than two more launches; few long rows are dealt out in parts (us, a
// workgroup / parts: one row of 50000 12.5 / 17.9, of 100000 18.5 / 17.7, of 250000 38 / 18; of 131072 64 rows 25 / 23, 128 rows 27 / 31).
constexpr int64_t kRowMost = 8 * kRowThreads;                    // vectors
constexpr int64_t kReadTwice = 12288;                            // vectors
constexpr int64_t kDistillRows = 112;
constexpr int64_t kDistillGroups = 512;

RowPlan part_plan(int64_t rows, int64_t vocab) {
    const int64_t vecs = (vocab + 14) / 8;
    const int64_t parts = std::max((vecs + kPartMost - 1) / kPartMost, std::min((kDistillGroups + rows - 1) / rows, (vecs + kPartThreads - 1) / kPartThreads));
    const int64_t each = (vecs + parts - 1) / parts;
    return {(uint32_t)((vecs + each - 1) / each), (uint32_t)each};
}

RowPlan distill_plan(int64_t rows, int64_t vocab) {
    const int64_t vecs = (vocab + 14) / 8;
    if (vecs <= kReadTwice || rows >= kDistillRows) return {1, (uint32_t)vecs};
    return part_plan(rows, vocab);
}

bool temperature_ok(double t) { return t > 0.0 && t >= 1e-6 && t <= 1e6; }

}  // namespace

extern "C" {

size_t sbc_mxfp_bytes(int64_t rows, int64_t cols) {
    if (!dim_ok(rows) || !dim_ok(cols)) return 0;
    return (size_t)(mx_panels(rows) * mx_steps(cols)) * (kMxPanelBytes + kMxScaleBytes);
}

int sbc_mxfp_quantize(int device, void* hip_stream, const void* x, int type, int64_t rows, int64_t cols, int64_t ld, void* by_rows, void* by_cols) {
    if (rows == 0 && dim_ok(cols) && size_of(type) && !by_cols) return SBC_OK;
    if (!dim_ok(rows) || !dim_ok(cols) || !dense_ok(x, type, cols, ld) || (!by_rows && !by_cols) || by_rows == by_cols) return SBC_EINVAL;
    if ((by_rows && !held_ok(by_rows)) || (by_cols && !held_ok(by_cols))) return SBC_EINVAL;
    if (!tiles_fit(rows, cols)) return SBC_ECAPACITY;
    if (!apart({held_span(by_rows, rows, cols), held_span(by_cols, cols, rows)}, {matrix_span(x, type, rows, cols, ld)})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    return by_type(type, [&](auto t) {
        launch_quantize<decltype(t)>(static_cast<hipStream_t>(hip_stream), x, rows, cols, ld, by_rows, by_cols);
        return launched();
    });
}

int sbc_mxfp_dequantize(int device, void* hip_stream, const void* q, int64_t rows, int64_t cols, void* y, int type, int64_t ld) {
    if (rows == 0 && dim_ok(cols) && size_of(type)) return SBC_OK;
    if (!dim_ok(rows) || !dim_ok(cols) || !held_ok(q) || !dense_ok(y, type, cols, ld)) return SBC_EINVAL;
    if (!tiles_fit(rows, cols)) return SBC_ECAPACITY;
    if (!apart({matrix_span(y, type, rows, cols, ld)}, {held_span(q, rows, cols)})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        const uint32_t steps = (uint32_t)mx_steps(cols);
        hipLaunchKernelGGL((k_mxfp_dequantize<T>), dim3((uint32_t)mx_panels(rows) * steps), dim3(256), 0, static_cast<hipStream_t>(hip_stream),
                           container(q, rows, cols), rows, cols, steps, static_cast<T*>(y), ld);
        return launched();
    });
}

int sbc_mxfp_matmul(int device, void* hip_stream, const void* a, const void* b, int64_t M, int64_t N, int64_t K, void* c, int type, int64_t ldc) {
    if (M == 0 && dim_ok(N) && dim_ok(K) && size_of(type)) return SBC_OK;
    if (!dim_ok(M) || !dim_ok(N) || !dim_ok(K) || !held_ok(a) || !held_ok(b) || !dense_ok(c, type, N, ldc)) return SBC_EINVAL;
    if (!product_fits(M, N)) return SBC_ECAPACITY;
    if (!apart({matrix_span(c, type, M, N, ldc)}, {held_span(a, M, K), held_span(b, N, K)})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        launch_product<T>(static_cast<hipStream_t>(hip_stream), container(a, M, K), container(b, N, K), M, N, K, static_cast<T*>(c), ldc);
        return launched();
    });
}

size_t sbc_mxfp_linear_workspace(int64_t M, int64_t K) { return dim_ok(M) && dim_ok(K) && few_values(M, K) <= kFewAlways ? 0 : sbc_mxfp_bytes(M, K); }

int sbc_mxfp_linear(int device, void* hip_stream, const void* x, int type, int64_t ldx, int64_t M, const void* w, int64_t N, int64_t K, void* y, int64_t ldy,
                    void* workspace, size_t workspace_bytes) {
    if (M == 0 && dim_ok(N) && dim_ok(K) && size_of(type)) return SBC_OK;
    if (!dim_ok(M) || !dim_ok(N) || !dim_ok(K) || !dense_ok(x, type, K, ldx) || !held_ok(w) || !dense_ok(y, type, N, ldy)) return SBC_EINVAL;
    const size_t room = sbc_mxfp_linear_workspace(M, K);
    if (room && !held_ok(workspace)) return SBC_EINVAL;
    if (workspace_bytes < room || !product_fits(M, N) || !tiles_fit(M, K)) return SBC_ECAPACITY;
    if (!apart({matrix_span(y, type, M, N, ldy), {workspace, room}}, {matrix_span(x, type, M, K, ldx), held_span(w, N, K)})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        if (few_fused(M, N, K)) {
            launch_few_tiles<T, 1, true>(stream, static_cast<const T*>(x), ldx, MxPtr{}, M, K, container(w, N, K), N, static_cast<T*>(y), ldy);
            return launched();
        }
        launch_quantize<T>(stream, x, M, K, ldx, workspace, nullptr);
        if (const int rc = launched()) return rc;
        launch_product<T>(stream, container(workspace, M, K), container(w, N, K), M, N, K, static_cast<T*>(y), ldy);
        return launched();
    });
}

size_t sbc_top_logits_workspace(int64_t rows, int64_t vocab, int k) {
    if (!dim_ok(rows) || !dim_ok(vocab) || k < 1 || k > SBC_TOP_MAX) return 0;
    return top_room(rows, vocab, k);
}

int sbc_top_logits(int device, void* hip_stream, const void* logits, int type, int64_t ld, int64_t rows, int64_t vocab, int k, double temperature,
                   int32_t* index, float* top, float* lse, void* workspace, size_t workspace_bytes) {
    if (k < 1 || k > SBC_TOP_MAX || !dim_ok(vocab) || !temperature_ok(temperature) || !size_of(type)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!dim_ok(rows) || !dense_ok(logits, type, vocab, ld) || !index || !top || !aligned(index, 4) || !aligned(top, 4) || !aligned(lse, 4)) return SBC_EINVAL;
    const size_t room = top_room(rows, vocab, k);
    if (room && (!workspace || !aligned(workspace, 16))) return SBC_EINVAL;
    if (workspace_bytes < room) return SBC_ECAPACITY;
    const uint64_t listed = (uint64_t)rows * k * 4;
    if (!apart({{index, listed}, {top, listed}, {lse, (uint64_t)rows * 4}, {workspace, room}}, {matrix_span(logits, type, rows, vocab, ld)})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const RowPlan p = top_plan(rows, vocab, k);
    const float inv_t = (float)(1.0 / temperature), c = (float)(1.4426950408889634 / temperature);
    ExpSum* const sums = static_cast<ExpSum*>(workspace);
    unsigned long long* const keys = reinterpret_cast<unsigned long long*>(sums + (room ? rows * p.parts : 0));
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        by_rows_of(rows, p.parts, [&](int64_t r, int64_t n) {
            const T* const x = static_cast<const T*>(logits) + r * ld;
            const TopOut out = {index + r * k, top + r * k, lse ? lse + r : nullptr};
            ExpSum* const pi = room ? sums + r * p.parts : nullptr;
            unsigned long long* const pk = room ? keys + (size_t)r * p.parts * k : nullptr;
            if (rows >= kTopManyRows && k <= kTopManyListed && p.vecs <= 2 * kTopThreads) launch_top<T, 4, 64>(stream, n * p.parts, x, ld, vocab, k, p, inv_t, c, out, pk, pi);
            else if (p.vecs <= 2 * kTopThreads) launch_top<T, 2, kTopThreads>(stream, n * p.parts, x, ld, vocab, k, p, inv_t, c, out, pk, pi);
            else launch_top<T, 4, kTopThreads>(stream, n * p.parts, x, ld, vocab, k, p, inv_t, c, out, pk, pi);
            if (p.parts > 1) hipLaunchKernelGGL(k_top_join, dim3((uint32_t)n), dim3(kJoinThreads), 0, stream, (uint32_t)k, p.parts, inv_t, c, out, pk, pi);
        });
        return launched();
    });
}

size_t sbc_distill_workspace(int64_t rows, int64_t vocab) {
    if (!dim_ok(rows) || !dim_ok(vocab)) return 0;
    const RowPlan p = distill_plan(rows, vocab);
    return p.parts == 1 ? 0 : (size_t)rows * (sizeof(DistillStats) + p.parts * sizeof(ExpSum));
}

}  // extern "C"

namespace {

bool distill_ok(const void* logits, int type, int64_t ld, int64_t rows, int64_t vocab, const int32_t* index, const float* top, int k, const float* teacher_lse,
                const float* weight) {
    return dim_ok(rows) && dense_ok(logits, type, vocab, ld) && index && top && aligned(index, 4) && aligned(top, 4) && aligned(teacher_lse, 4) && aligned(weight, 4) &&
           k >= 1 && k <= SBC_TOP_MAX;
}

DistillArgs distill_args(const int32_t* index, const float* top, const float* teacher_lse, const float* weight, int k, double temperature) {
    return {index, top, teacher_lse, weight, (uint32_t)k, (float)(1.4426950408889634 / temperature), (float)temperature, 1.0 / temperature};
}

// ... of the rows from r on
DistillArgs from_row(DistillArgs a, int64_t r) {
    a.index += r * a.k;
    a.top += r * a.k;
    if (a.teacher_lse) a.teacher_lse += r;
    if (a.weight) a.weight += r;
    return a;
}

template <typename T>
void launch_grad(hipStream_t stream, const T* logits, int64_t ld, int64_t rows, int64_t vocab, const DistillArgs& args, const DistillStats* stats, T* grad, int64_t ld_grad) {
    const RowPlan p = part_plan(rows, vocab);
    by_rows_of(rows, p.parts, [&](int64_t r, int64_t n) {
        hipLaunchKernelGGL((k_distill_grad<T>), dim3((uint32_t)(n * p.parts)), dim3(kPartThreads + 64), 0, stream, logits + r * ld, ld, (uint32_t)vocab, from_row(args, r),
                           stats + r, p.parts, p.vecs, grad + r * ld_grad, ld_grad);
    });
}

template <typename T, int n, int threads>
void launch_row(hipStream_t stream, const T* logits, int64_t ld, int64_t rows, int64_t vocab, const DistillArgs& args, const DistillOut& out, T* grad, int64_t ld_grad) {
    hipLaunchKernelGGL((k_distill_row<T, n, threads>), dim3((uint32_t)rows), dim3(threads + 64), 0, stream, logits, ld, (uint32_t)vocab, args, out, grad, ld_grad);
}

// Workgroups of as few wavefronts as hold the row: a row's steps wait for one another, so that it is the rows under way that
// count (us, this / 512 threads for all: 700 x 10000 14.3 / 18.3, 1600 x 5000 18.3 / 25.3; up to 300 rows alike).
template <typename T>
void launch_rows(hipStream_t stream, int64_t vecs, const T* x, int64_t ld, int64_t rows, int64_t vocab, const DistillArgs& a, const DistillOut& out, T* g, int64_t ldg) {
    if (vecs <= 128) launch_row<T, 1, 128>(stream, x, ld, rows, vocab, a, out, g, ldg);
    else if (vecs <= 256) launch_row<T, 2, 128>(stream, x, ld, rows, vocab, a, out, g, ldg);
    else if (vecs <= 512) launch_row<T, 4, 128>(stream, x, ld, rows, vocab, a, out, g, ldg);
    else if (vecs <= 1024) launch_row<T, 4, 256>(stream, x, ld, rows, vocab, a, out, g, ldg);
    else if (vecs <= 1536) launch_row<T, 6, 256>(stream, x, ld, rows, vocab, a, out, g, ldg);
    else if (vecs <= 2048) launch_row<T, 4, 512>(stream, x, ld, rows, vocab, a, out, g, ldg);
    else launch_row<T, 8, 512>(stream, x, ld, rows, vocab, a, out, g, ldg);
}

}  // namespace

extern "C" {

int sbc_distill_loss(int device, void* hip_stream, const void* logits, int type, int64_t ld, int64_t rows, int64_t vocab, const int32_t* index, const float* top, int k,
                     const float* teacher_lse, double temperature, const float* weight, float* loss, float* stats, void* grad, int64_t ld_grad,
                     void* workspace, size_t workspace_bytes) {
    if (k < 1 || k > SBC_TOP_MAX || !dim_ok(vocab) || !temperature_ok(temperature) || !size_of(type)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!distill_ok(logits, type, ld, rows, vocab, index, top, k, teacher_lse, weight) || !loss || !aligned(loss, 4) || !aligned(stats, 16)) return SBC_EINVAL;
    if (grad && (!dense_ok(grad, type, vocab, ld_grad) || (grad == logits && ld_grad != ld))) return SBC_EINVAL;
    const size_t room = sbc_distill_workspace(rows, vocab);
    if (room && (!workspace || !aligned(workspace, 16))) return SBC_EINVAL;
    if (workspace_bytes < room) return SBC_ECAPACITY;
    const uint64_t listed = (uint64_t)rows * k * 4, each = (uint64_t)rows * 4;
    // (in place the logits are what is written)
    if (!apart({{loss, each}, {stats, 4 * each}, {workspace, room}, matrix_span(grad, type, rows, vocab, ld_grad)},
               {matrix_span(grad == logits ? nullptr : logits, type, rows, vocab, ld), {index, listed}, {top, listed}, {teacher_lse, each}, {weight, each}})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const DistillArgs args = distill_args(index, top, teacher_lse, weight, k, temperature);
    const RowPlan p = distill_plan(rows, vocab);
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        const T* const x = static_cast<const T*>(logits);
        T* const g = static_cast<T*>(grad);
        DistillStats* const st = reinterpret_cast<DistillStats*>(stats);
        if (p.parts == 1) {
            by_rows_of(rows, 1, [&](int64_t r, int64_t n) {
                const DistillArgs a = from_row(args, r);
                const DistillOut out = {loss + r, st ? st + r : nullptr};
                T* const gr = g ? g + r * ld_grad : nullptr;
                const T* const xr = x + r * ld;
                if (p.vecs <= kRowMost) launch_rows<T>(stream, p.vecs, xr, ld, n, vocab, a, out, gr, ld_grad);
                else hipLaunchKernelGGL((k_distill<T>), dim3((uint32_t)n), dim3(kRowThreads), 0, stream, xr, ld, (uint32_t)vocab, a, out, gr, ld_grad);
            });
            return launched();
        }
        DistillStats* const own = st ? st : static_cast<DistillStats*>(workspace);
        ExpSum* const sums = reinterpret_cast<ExpSum*>(static_cast<DistillStats*>(workspace) + rows);
        const DistillOut out = {loss, own};
        hipLaunchKernelGGL((k_distill_part<T>), dim3((uint32_t)(rows * p.parts)), dim3(kPartThreads), 0, stream, x, ld, (uint32_t)vocab, args, p.parts, p.vecs, sums);
        hipLaunchKernelGGL((k_distill_join<T>), dim3((uint32_t)rows), dim3(64), 0, stream, x, ld, (uint32_t)vocab, args, p.parts, sums, out);
        if (g) launch_grad<T>(stream, x, ld, rows, vocab, args, own, g, ld_grad);
        return launched();
    });
}

int sbc_distill_grad(int device, void* hip_stream, const void* logits, int type, int64_t ld, int64_t rows, int64_t vocab, const int32_t* index, const float* top, int k,
                     const float* teacher_lse, double temperature, const float* stats, const float* dloss, void* grad, int64_t ld_grad) {
    if (k < 1 || k > SBC_TOP_MAX || !dim_ok(vocab) || !temperature_ok(temperature) || !size_of(type)) return SBC_EINVAL;
    if (rows == 0) return SBC_OK;
    if (!distill_ok(logits, type, ld, rows, vocab, index, top, k, teacher_lse, dloss) || !stats || !aligned(stats, 16)) return SBC_EINVAL;
    if (!dense_ok(grad, type, vocab, ld_grad) || (grad == logits && ld_grad != ld)) return SBC_EINVAL;
    const uint64_t listed = (uint64_t)rows * k * 4, each = (uint64_t)rows * 4;
    if (!apart({matrix_span(grad, type, rows, vocab, ld_grad)},
               {matrix_span(grad == logits ? nullptr : logits, type, rows, vocab, ld), {index, listed}, {top, listed}, {teacher_lse, each}, {stats, 4 * each}, {dloss, each}})) return SBC_EINVAL;
    if (const int rc = device_status(device)) return rc;
    DeviceScope scope(device);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const DistillArgs args = distill_args(index, top, teacher_lse, dloss, k, temperature);
    return by_type(type, [&](auto t) {
        typedef decltype(t) T;
        launch_grad<T>(stream, static_cast<const T*>(logits), ld, rows, vocab, args, reinterpret_cast<const DistillStats*>(stats), static_cast<T*>(grad), ld_grad);
        return launched();
    });
}

}  // extern "C"
