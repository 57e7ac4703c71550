// Entry points of the operators on messages and logits: checks of what the caller gives.  No allocation, no exception.
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "dsq_answers.h"

namespace {

constexpr uint64_t kMost = 1ull << 31, kMostSide = 1ull << 28;   // of a matrix: 32 rows apart is less than 2^32 bytes

struct Report {
    char* buf;
    uint64_t len;
    ds_status operator()(ds_status st, const char* format, ...) const {
        if (buf && len) {
            va_list args;
            va_start(args, format);
            std::vsnprintf(buf, (size_t)len, format, args);
            va_end(args);
        }
        return st;
    }
    ds_status done(hipError_t e) const {
        if (e != hipSuccess) return (*this)(DS_EHIP, "launching the kernel failed: %s", hipGetErrorString(e));
        return (*this)(DS_OK, "%s", "");
    }
};

uint64_t address(const void* p) { return (uint64_t)reinterpret_cast<uintptr_t>(p); }
uint64_t size_of(int32_t dtype) { return dtype == DS_F32 ? 4 : 2; }
bool known(int32_t dtype) { return dtype == DS_F32 || dtype == DS_BF16 || dtype == DS_F16; }

const char* matrix_fault(const ds_matrix* m) {
    if (!m) return "the matrix is NULL";
    if (m->rows < 1 || m->rows >= kMostSide) return "rows must be at least 1 and below 2^28";
    if (m->cols < 1 || m->cols >= kMostSide) return "cols must be at least 1 and below 2^28";
    if (m->block < 64 || m->block > 2048 || (m->block & (m->block - 1))) return "block must be a power of two between 64 and 2048";
    return nullptr;
}

const char* product_fault(const ds_matrix* m) {
    if (const char* why = matrix_fault(m)) return why;
    if (m->tokens >= kMost) return "tokens must be below 2^31";
    if (!known(m->dtype)) return "unknown dtype";
    return nullptr;
}

const char* logits_fault(const ds_logits* l) {
    if (!l) return "the logits' description is NULL";
    if (l->rows >= kMost) return "rows must be below 2^31";
    if (l->vocab < 1 || l->vocab >= kMost) return "vocab must be at least 1 and below 2^31";
    if (l->k < 1 || l->k > dsq::kMaxTop) return "k must be between 1 and 256";
    if (!known(l->dtype)) return "unknown dtype";
    if (!std::isfinite(l->temperature) || !(l->temperature >= FLT_MIN)) return "temperature must be finite and positive, and no subnormal number";
    if (l->reserved != 0) return "reserved must be 0";
    return nullptr;
}

uint64_t row_bytes(const ds_matrix& m) {
    const uint64_t block = (uint64_t)m.block, full = m.cols / block, tail = m.cols % block;
    return full * (4 + block / 2) + (tail ? 4 + 4 * ((tail + 7) / 8) : 0);
}

// The address range of `rows` rows of `width` elements with pitch ld; false if it does not fit into 64 bits.
bool range(const void* p, uint64_t rows, uint64_t width, uint64_t ld, uint64_t size, uint64_t& lo, uint64_t& hi) {
    unsigned __int128 bytes = ((unsigned __int128)(rows - 1) * ld + width) * size;
    lo = address(p);
    if (bytes > (unsigned __int128)(UINT64_MAX - lo)) return false;
    hi = lo + (uint64_t)bytes;
    return true;
}

ds_status check_work(const Report& report, const void* work, uint64_t given, uint64_t needed) {
    if (needed == 0) return DS_OK;
    if (!work || given < needed)
        return report(DS_EINVAL, "work_dev: %llu bytes are needed, %llu given", (unsigned long long)needed, (unsigned long long)(work ? given : 0));
    if (address(work) & 15) return report(DS_EINVAL, "work_dev must be 16-byte aligned");
    return DS_OK;
}

// Both products: `in` has in_width columns, `out` out_width.
ds_status product_call(const ds_matrix* m, const void* msg, const void* in, uint64_t in_ld, uint64_t in_width, void* out, uint64_t out_ld,
                       uint64_t out_width, void* work, uint64_t given, uint64_t needed, const Report& report, dsq::ProductArgs& a) {
    if (!msg || !in || !out) return report(DS_EINVAL, "a device pointer is NULL");
    if (in_ld < in_width || out_ld < out_width) return report(DS_EINVAL, "a pitch is smaller than the row it holds");
    const uint64_t size = size_of(m->dtype);
    if (address(msg) & 3) return report(DS_EINVAL, "msg_dev must be 4-byte aligned");
    if ((address(in) | address(out)) & (size - 1)) return report(DS_EINVAL, "inputs and outputs must be aligned to their elements");
    uint64_t in_lo, in_hi, out_lo, out_hi, msg_lo, msg_hi;
    if (!range(in, m->tokens, in_width, in_ld, size, in_lo, in_hi) || !range(out, m->tokens, out_width, out_ld, size, out_lo, out_hi) ||
        !range(msg, m->rows, row_bytes(*m), row_bytes(*m), 1, msg_lo, msg_hi))
        return report(DS_EINVAL, "an array does not fit into the address space");
    if ((out_lo < in_hi && in_lo < out_hi) || (out_lo < msg_hi && msg_lo < out_hi)) return report(DS_EINVAL, "the output overlaps an input");
    if (const ds_status st = check_work(report, work, given, needed)) return st;
    a.msg = static_cast<const uint8_t*>(msg);
    a.in = in; a.out = out; a.work = work;
    a.rows = m->rows; a.cols = m->cols; a.tokens = m->tokens;
    a.in_ld = in_ld; a.out_ld = out_ld;
    a.row_bytes = row_bytes(*m);
    a.block = (uint32_t)m->block;
    a.dtype = m->dtype;
    return DS_OK;
}

ds_status logits_call(const ds_logits* l, const void* z, uint64_t z_ld, const void* pairs, const Report& report, dsq::LogitsArgs& a) {
    if (!z || !pairs) return report(DS_EINVAL, "a device pointer is NULL");
    if (z_ld < l->vocab) return report(DS_EINVAL, "z_ld must be >= vocab");
    const uint64_t size = size_of(l->dtype);
    if (address(z) & (size - 1)) return report(DS_EINVAL, "z_dev must be aligned to its elements");
    if (address(pairs) & 7) return report(DS_EINVAL, "pairs_dev must be 8-byte aligned");
    uint64_t lo, hi;
    if (!range(z, l->rows, l->vocab, z_ld, size, lo, hi)) return report(DS_EINVAL, "z does not fit into the address space");
    a.z = z; a.z_ld = z_ld;
    a.rows = l->rows; a.vocab = l->vocab; a.k = (uint32_t)l->k; a.dtype = l->dtype; a.temperature = l->temperature;
    return DS_OK;
}

}  // namespace

extern "C" {

uint64_t ds_matrix_bytes(const ds_matrix* m) { return matrix_fault(m) ? 0 : m->rows * row_bytes(*m); }

uint64_t ds_product_work_bytes(const ds_matrix* m) { return product_fault(m) || m->tokens == 0 ? 0 : dsq::product_work_bytes(*m); }

uint64_t ds_product_gradient_work_bytes(const ds_matrix* m) {
    return product_fault(m) || m->tokens == 0 ? 0 : dsq::product_gradient_work_bytes(*m);
}

uint64_t ds_top_logits_work_bytes(const ds_logits* l) { return logits_fault(l) || l->rows == 0 ? 0 : dsq::top_logits_work_bytes(*l); }

uint64_t ds_distill_work_bytes(const ds_logits* l) { return logits_fault(l) || l->rows == 0 ? 0 : dsq::distill_work_bytes(*l); }

ds_status ds_product(const ds_matrix* m, const void* msg_dev, const void* x_dev, uint64_t x_ld, void* y_dev, uint64_t y_ld,
                     void* work_dev, uint64_t work_bytes, void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = product_fault(m)) return report(DS_EINVAL, "%s", why);
    if (m->tokens == 0) return report(DS_OK, "%s", "");
    dsq::ProductArgs a{};
    if (const ds_status st = product_call(m, msg_dev, x_dev, x_ld, m->cols, y_dev, y_ld, m->rows, work_dev, work_bytes,
                                          dsq::product_work_bytes(*m), report, a))
        return st;
    return report.done(dsq::launch_product(a, static_cast<hipStream_t>(hip_stream)));
}

ds_status ds_product_gradient(const ds_matrix* m, const void* msg_dev, const void* dy_dev, uint64_t dy_ld, void* dx_dev,
                              uint64_t dx_ld, void* work_dev, uint64_t work_bytes, void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = product_fault(m)) return report(DS_EINVAL, "%s", why);
    if (m->tokens == 0) return report(DS_OK, "%s", "");
    dsq::ProductArgs a{};
    if (const ds_status st = product_call(m, msg_dev, dy_dev, dy_ld, m->rows, dx_dev, dx_ld, m->cols, work_dev, work_bytes,
                                          dsq::product_gradient_work_bytes(*m), report, a))
        return st;
    return report.done(dsq::launch_product_gradient(a, static_cast<hipStream_t>(hip_stream)));
}

ds_status ds_top_logits(const ds_logits* l, const void* z_dev, uint64_t z_ld, void* pairs_dev, float* lse_dev, void* work_dev,
                        uint64_t work_bytes, void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = logits_fault(l)) return report(DS_EINVAL, "%s", why);
    if ((uint64_t)l->k > l->vocab) return report(DS_EINVAL, "k must not exceed vocab");
    if (l->rows == 0) return report(DS_OK, "%s", "");
    dsq::LogitsArgs a{};
    if (const ds_status st = logits_call(l, z_dev, z_ld, pairs_dev, report, a)) return st;
    if (address(lse_dev) & 3) return report(DS_EINVAL, "lse_dev must be 4-byte aligned");
    if (const ds_status st = check_work(report, work_dev, work_bytes, dsq::top_logits_work_bytes(*l))) return st;
    a.pairs = static_cast<uint2*>(pairs_dev);
    a.lse = lse_dev;
    a.work = work_dev;
    return report.done(dsq::launch_top_logits(a, static_cast<hipStream_t>(hip_stream)));
}

ds_status ds_distill(const ds_logits* l, const void* z_dev, uint64_t z_ld, const void* pairs_dev, const float* teacher_lse_dev,
                     const float* weight_dev, float* loss_dev, void* dz_dev, uint64_t dz_ld, void* work_dev, uint64_t work_bytes,
                     void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = logits_fault(l)) return report(DS_EINVAL, "%s", why);
    if (l->rows == 0) return report(DS_OK, "%s", "");
    dsq::LogitsArgs a{};
    if (const ds_status st = logits_call(l, z_dev, z_ld, pairs_dev, report, a)) return st;
    if (!loss_dev && !dz_dev) return report(DS_EINVAL, "neither a loss nor a gradient is asked for");
    if ((address(teacher_lse_dev) | address(weight_dev) | address(loss_dev)) & 3) return report(DS_EINVAL, "an array of floats must be 4-byte aligned");
    if (dz_dev) {
        const uint64_t size = size_of(l->dtype);
        if (dz_ld < l->vocab) return report(DS_EINVAL, "dz_ld must be >= vocab");
        if (address(dz_dev) & (size - 1)) return report(DS_EINVAL, "dz_dev must be aligned to its elements");
        uint64_t z_lo, z_hi, dz_lo, dz_hi;
        if (!range(dz_dev, l->rows, l->vocab, dz_ld, size, dz_lo, dz_hi)) return report(DS_EINVAL, "dz does not fit into the address space");
        (void)range(z_dev, l->rows, l->vocab, z_ld, size, z_lo, z_hi);
        if (!(dz_dev == z_dev && dz_ld == z_ld) && dz_lo < z_hi && z_lo < dz_hi)
            return report(DS_EINVAL, "dz overlaps z without being it (same address, same pitch)");
    }
    if (const ds_status st = check_work(report, work_dev, work_bytes, dsq::distill_work_bytes(*l))) return st;
    a.given = static_cast<const uint2*>(pairs_dev);
    a.teacher_lse = teacher_lse_dev; a.weight = weight_dev;
    a.loss = loss_dev; a.dz = dz_dev; a.dz_ld = dz_ld;
    a.work = work_dev;
    return report.done(dsq::launch_distill(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
