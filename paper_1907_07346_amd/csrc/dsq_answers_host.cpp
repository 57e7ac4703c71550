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

const char* sampling_fault(const ds_sampling* s) {
    if (!s) return "the sampling's description is NULL";
    if (s->rows >= kMost) return "rows must be below 2^31";
    if (s->vocab < 1 || s->vocab >= kMost) return "vocab must be at least 1 and below 2^31";
    if (!known(s->dtype)) return "unknown dtype";
    if (s->top_k < 0) return "top_k must not be negative";
    if (!(s->temperature == 0.f || (std::isfinite(s->temperature) && s->temperature >= FLT_MIN)))
        return "temperature must be 0, or finite and positive, and no subnormal number";
    if (!(s->top_p >= 0.f && s->top_p <= 1.f)) return "top_p must be between 0 and 1";
    if (!(s->min_p >= 0.f && s->min_p <= 1.f)) return "min_p must be between 0 and 1";
    if (s->reserved != 0) return "reserved must be 0";
    return nullptr;
}

// What is wrong with a list of tensors, and the numbers that go into its ds_gradients.
const char* tensors_fault(const ds_tensor* tensors, uint64_t count, uint64_t workers, ds_gradients& g) {
    if (workers < 1 || workers >= (1ull << 20)) return "workers must be at least 1 and below 2^20";
    if (count >= (1ull << 24)) return "there must be fewer than 2^24 tensors";
    if (count && !tensors) return "the list of tensors is NULL";
    g = ds_gradients{};
    g.workers = workers;
    g.tensors = count;
    uint64_t column = 0, tiles = 0;
    int32_t before = 0;
    for (uint64_t i = 0; i < count; ++i) {
        const ds_tensor& t = tensors[i];
        if (t.worker < before || (uint64_t)t.worker >= workers) return "the tensors' workers must not descend and must be below `workers`";
        if (!known(t.dtype)) return "unknown dtype";
        if (t.count >= (1ull << 40)) return "a tensor must have fewer than 2^40 elements";
        const uint64_t size = size_of(t.dtype);
        if (t.count && !t.data_dev) return "a device pointer is NULL";
        if (t.count && (address(t.data_dev) & (size - 1))) return "tensors must be aligned to their elements";
        if (t.count && address(t.data_dev) > UINT64_MAX - t.count * size) return "a tensor does not fit into the address space";
        if (t.worker != before) column = tiles = 0;
        before = t.worker;
        column += t.count;
        if (column >= (1ull << 40)) return "a worker must have fewer than 2^40 elements";
        const uint64_t of = (t.count + dsq::kGradientTile - 1) / dsq::kGradientTile;
        tiles += of;
        g.tiles += of;
        if (g.tiles >= (1ull << 32) - 1) return "too many elements";
        if (column > g.columns) g.columns = column;
        if (tiles > g.worker_tiles) g.worker_tiles = tiles;
    }
    g.table_bytes = dsq::gradients_table_bytes(workers, count, g.tiles);
    return nullptr;
}

const char* gradients_fault(const ds_gradients* g) {
    if (!g) return "the gradients' description is NULL";
    if (!g->table_dev || (address(g->table_dev) & 15) || g->workers < 1 || g->workers >= (1ull << 20) || g->tensors >= (1ull << 24) ||
        g->tiles >= (1ull << 32) - 1 || g->worker_tiles > g->tiles || g->table_bytes != dsq::gradients_table_bytes(g->workers, g->tensors, g->tiles))
        return "the gradients' description is not what ds_gradients_lay made";
    return nullptr;
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

uint64_t ds_sample_work_bytes(const ds_sampling* s) { return sampling_fault(s) || s->rows == 0 ? 0 : dsq::sample_work_bytes(*s); }

ds_status ds_sample(const ds_sampling* s, const ds_sampling_rows* each, const void* z_dev, uint64_t z_ld, const float* u_dev,
                    int32_t* token_dev, float* logp_dev, void* work_dev, uint64_t work_bytes, void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = sampling_fault(s)) return report(DS_EINVAL, "%s", why);
    if (s->rows == 0) return report(DS_OK, "%s", "");
    if (!z_dev || !u_dev || !token_dev) return report(DS_EINVAL, "a device pointer is NULL");
    if (z_ld < s->vocab) return report(DS_EINVAL, "z_ld must be >= vocab");
    if (address(z_dev) & (size_of(s->dtype) - 1)) return report(DS_EINVAL, "z_dev must be aligned to its elements");
    const ds_sampling_rows own = each ? *each : ds_sampling_rows{};
    if ((address(u_dev) | address(token_dev) | address(logp_dev) | address(own.temperature_dev) | address(own.top_k_dev) | address(own.top_p_dev) |
         address(own.min_p_dev)) & 3)
        return report(DS_EINVAL, "an array of a number per row must be 4-byte aligned");
    uint64_t z_lo, z_hi;
    if (!range(z_dev, s->rows, s->vocab, z_ld, size_of(s->dtype), z_lo, z_hi)) return report(DS_EINVAL, "z does not fit into the address space");
    // outputs are neither inputs nor each other
    const void* const arrays[] = {token_dev, logp_dev, u_dev, own.temperature_dev, own.top_k_dev, own.top_p_dev, own.min_p_dev};
    for (int i = 0; i < 2; ++i) {
        uint64_t lo, hi, other_lo, other_hi;
        if (!arrays[i]) continue;
        if (!range(arrays[i], 1, s->rows, s->rows, 4, lo, hi)) return report(DS_EINVAL, "an array does not fit into the address space");
        if (lo < z_hi && z_lo < hi) return report(DS_EINVAL, "an output overlaps z");
        for (int j = i + 1; j < 7; ++j) {
            if (!arrays[j]) continue;
            if (!range(arrays[j], 1, s->rows, s->rows, 4, other_lo, other_hi)) return report(DS_EINVAL, "an array does not fit into the address space");
            if (lo < other_hi && other_lo < hi) return report(DS_EINVAL, "an output overlaps another array");
        }
    }
    if (const ds_status st = check_work(report, work_dev, work_bytes, dsq::sample_work_bytes(*s))) return st;
    dsq::SampleArgs a{};
    a.z = z_dev; a.z_ld = z_ld;
    a.rows = s->rows; a.vocab = s->vocab; a.dtype = s->dtype;
    a.top_k = s->top_k; a.temperature = s->temperature; a.top_p = s->top_p; a.min_p = s->min_p;
    a.each = own;
    a.u = u_dev; a.token = token_dev; a.logp = logp_dev; a.work = work_dev;
    return report.done(dsq::launch_sample(a, static_cast<hipStream_t>(hip_stream)));
}

uint64_t ds_gradients_bytes(const ds_tensor* tensors, uint64_t count, uint64_t workers) {
    ds_gradients g;
    return tensors_fault(tensors, count, workers, g) ? 0 : g.table_bytes;
}

ds_status ds_gradients_lay(const ds_tensor* tensors, uint64_t count, uint64_t workers, void* table_dev, uint64_t table_bytes,
                           ds_gradients* out, void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    ds_gradients g;
    if (const char* why = tensors_fault(tensors, count, workers, g)) return report(DS_EINVAL, "%s", why);
    if (!out) return report(DS_EINVAL, "out is NULL");
    if (!table_dev || table_bytes < g.table_bytes)
        return report(DS_EINVAL, "table_dev: %llu bytes are needed, %llu given", (unsigned long long)g.table_bytes, (unsigned long long)(table_dev ? table_bytes : 0));
    if (address(table_dev) & 15) return report(DS_EINVAL, "table_dev must be 16-byte aligned");
    g.table_dev = table_dev;
    dsq::RecordBatch batch{};
    uint64_t column = 0, tile = 0, next_worker = 0;               // (workers before next_worker know their first tile)
    int32_t before = 0;
    for (uint64_t i = 0; i <= count; ++i) {
        dsq::TensorRecord& r = batch.record[batch.here++];
        if (i < count) {
            const ds_tensor& t = tensors[i];
            if (t.worker != before) column = 0;
            before = t.worker;
            r = {t.data_dev, t.count, column, tile, (uint32_t)t.dtype, (uint32_t)t.worker, next_worker};
            column += t.count;
            tile += (t.count + dsq::kGradientTile - 1) / dsq::kGradientTile;
        } else {
            r = {nullptr, 0, 0, tile, (uint32_t)DS_F32, (uint32_t)workers, next_worker};
        }
        next_worker = (uint64_t)r.worker + 1;
        if (batch.here == dsq::RecordBatch::kMost || i == count) {
            const hipError_t e = dsq::launch_lay(g, batch, static_cast<hipStream_t>(hip_stream));
            if (e != hipSuccess) return report.done(e);
            batch.first += batch.here;
            batch.here = 0;
        }
    }
    *out = g;
    return report.done(hipSuccess);
}

uint64_t ds_gradient_norm_work_bytes(const ds_gradients* g) { return gradients_fault(g) ? 0 : dsq::gradient_norm_work_bytes(*g); }

uint64_t ds_clip_work_bytes(const ds_gradients* g) { return gradients_fault(g) ? 0 : dsq::clip_work_bytes(*g); }

ds_status ds_gradient_norm(const ds_gradients* g, float* norm_dev, void* work_dev, uint64_t work_bytes, void* hip_stream, char* errbuf,
                           uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = gradients_fault(g)) return report(DS_EINVAL, "%s", why);
    if (!norm_dev) return report(DS_EINVAL, "a device pointer is NULL");
    if (address(norm_dev) & 3) return report(DS_EINVAL, "norm_dev must be 4-byte aligned");
    if (const ds_status st = check_work(report, work_dev, work_bytes, dsq::gradient_norm_work_bytes(*g))) return st;
    dsq::ClipArgs a{};
    a.g = *g;
    a.norm = norm_dev;
    a.work = work_dev;
    return report.done(dsq::launch_gradient_norm(a, static_cast<hipStream_t>(hip_stream)));
}

ds_status ds_clip(const ds_gradients* g, double max_norm, float* g_dev, uint64_t g_ld, float* norm_dev, void* work_dev, uint64_t work_bytes,
                  void* hip_stream, char* errbuf, uint64_t errbuf_len) {
    const Report report{errbuf, errbuf_len};
    if (const char* why = gradients_fault(g)) return report(DS_EINVAL, "%s", why);
    if (!(max_norm >= 0.0)) return report(DS_EINVAL, "max_norm must be a number that is not negative");
    if ((address(norm_dev) | address(g_dev)) & 3) return report(DS_EINVAL, "an array of floats must be 4-byte aligned");
    if (g_dev) {
        if (g_ld < g->columns) return report(DS_EINVAL, "g_ld must be at least %llu, the elements of the largest worker", (unsigned long long)g->columns);
        uint64_t lo, hi;
        if (!range(g_dev, g->workers, g->columns, g_ld, 4, lo, hi)) return report(DS_EINVAL, "g does not fit into the address space");
        const uint64_t table = address(g->table_dev);
        if (lo < table + g->table_bytes && table < hi) return report(DS_EINVAL, "g overlaps the table");
    }
    if (const ds_status st = check_work(report, work_dev, work_bytes, dsq::clip_work_bytes(*g))) return st;
    dsq::ClipArgs a{};
    a.g = *g;
    a.max_norm = max_norm;
    a.out = g_dev;
    a.out_ld = g_ld;
    a.norm = norm_dev;
    a.work = work_dev;
    return report.done(dsq::launch_clip(a, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
