// Host side of include/aed_vocab.h: argument checks and launches of the operators on rows of logits.
#include "../../include/aed_vocab.h"

#include <cmath>

#include "host_calls.h"
#include "vocab.h"

namespace {

using aed::fail;
using aed::finish;
using aed::guarded;
using aed::hip_status;

constexpr int64_t kMostStride = (int64_t)1 << 38;  // elements; in bytes and times the rows (2^22) at most 2^62

template <typename C> aed_status check_config(const C* c, const void* out) {
    if (!c || !out) return fail(AED_EINVAL, "cfg / out is NULL");
    if (c->struct_size != sizeof(C)) return fail(AED_EINVAL, "struct_size %u, expected %zu", c->struct_size, sizeof(C));
    if (c->vocab < 1) return fail(AED_EINVAL, "vocab must be >= 1");
    if (c->dtype != 0 && c->dtype != 1) return fail(AED_EINVAL, "dtype must be 0 or 1");
    if (c->vocab > aed::kMostVocab) return fail(AED_EUNSUPPORTED, "vocab %d is above %d", c->vocab, aed::kMostVocab);
    return AED_OK;
}
template <typename C> aed_status check_list(const C* c) {
    if (c->top < 1) return fail(AED_EINVAL, "top must be >= 1");
    if (!(c->temperature > 0.f) || !std::isfinite(c->temperature)) return fail(AED_EINVAL, "temperature must be a finite number > 0");
    if (c->temperature < 1e-20f || c->temperature > 1e20f) return fail(AED_EUNSUPPORTED, "temperature %g is not in 1e-20 to 1e20", (double)c->temperature);
    if (c->top > aed::kMostTop) return fail(AED_EUNSUPPORTED, "top %d is above %d", c->top, aed::kMostTop);
    return AED_OK;
}

// A handle: its configuration and its stream
template <typename C> struct Plan {
    C cfg;
    hipStream_t stream;
};
template <typename P, typename C> aed_status create(const C* cfg, void* hip_stream, P** out) {
    return guarded([&] {
        *out = new P;
        (*out)->cfg = *cfg;
        (*out)->stream = static_cast<hipStream_t>(hip_stream);
        return AED_OK;
    });
}

aed_status check_rows(const void* data, const char* name, int64_t stride, int32_t rows, int32_t vocab, int dtype) {
    if (!data) return fail(AED_EINVAL, "%s is NULL", name);
    if ((uintptr_t)data % (dtype == 1 ? 2 : 4) != 0) return fail(AED_EINVAL, "%s are not aligned to their elements", name);
    if (rows > 1 && (stride < vocab || stride > kMostStride))
        return fail(AED_EINVAL, "%s: %lld elements between rows; vocab (%d) to 2^38 are possible", name, (long long)stride, vocab);
    return AED_OK;
}
// no rows: nothing is looked at but their number
template <typename C> aed_status to_rows(const C& c, const void* logits, int64_t stride, int32_t rows, aed::LogitRows& to) {
    if (rows < 0) return fail(AED_EINVAL, "rows = %d", rows);
    if (rows > aed::kMostRows) return fail(AED_EUNSUPPORTED, "more than 2^22 - 1 rows");
    to = aed::LogitRows{logits, rows > 1 ? stride : 0, rows, c.vocab};
    return rows == 0 ? AED_OK : check_rows(logits, "logits", stride, rows, c.vocab, c.dtype);
}
// pointers to 32-bit elements, of which the first `need` have to be there
template <size_t N> aed_status check_words(const char* names, const void* const (&p)[N], size_t need) {
    for (size_t i = 0; i < N; ++i) {
        if (i < need && !p[i]) return fail(AED_EINVAL, "one of %s is NULL", names);
        if ((uintptr_t)p[i] % 4 != 0) return fail(AED_EINVAL, "one of %s is not aligned to 4 bytes", names);
    }
    return AED_OK;
}

constexpr double kLog2e = 1.4426950408889634074;
void set_temperature(const aed_distill_config& c, aed::DistillArgs& a) {
    const double t = c.temperature;
    a.top = c.top;
    a.temperature = c.temperature;
    a.scale_d = kLog2e / t;
    a.scale = (float)a.scale_d;
    if ((double)a.scale >= a.scale_d) a.scale = std::nextafter(a.scale, 0.f);
    a.scale_low = (float)(a.scale_d - (double)a.scale);  // above 2^-100, as the temperature is limited
    a.factor = t * t / kLog2e;
}

}  // namespace

struct aed_sampler : Plan<aed_sampler_config> {};
struct aed_top : Plan<aed_top_config> {};
struct aed_distill : Plan<aed_distill_config> {};

extern "C" {

aed_status aed_sampler_create(const aed_sampler_config* cfg, void* hip_stream, aed_sampler** out) {
    if (out) *out = nullptr;
    const aed_status st = check_config(cfg, out);
    return st == AED_OK ? create(cfg, hip_stream, out) : st;
}
aed_status aed_sampler_destroy(aed_sampler* plan) { return finish(plan); }

aed_status aed_sample(aed_sampler* p, const void* logits, int64_t row_stride, int32_t rows, const float* uniforms, const aed_sampling* how, int32_t* tokens,
                      float* logp) {
    if (!p || !how) return fail(AED_EINVAL, "plan / how is NULL");
    if (how->struct_size != sizeof(aed_sampling)) return fail(AED_EINVAL, "struct_size %u, expected %zu", how->struct_size, sizeof(aed_sampling));
    if (!(how->temperature >= 0.f) || !std::isfinite(how->temperature)) return fail(AED_EINVAL, "temperature must be a finite number >= 0");
    if (how->top_k < 0) return fail(AED_EINVAL, "top_k must be >= 0");
    if (!(how->top_p >= 0.f && how->top_p <= 1.f)) return fail(AED_EINVAL, "top_p must be in [0, 1]");
    if (!(how->min_p >= 0.f && how->min_p <= 1.f)) return fail(AED_EINVAL, "min_p must be in [0, 1]");
    aed::SampleArgs a = {};
    aed_status st = to_rows(p->cfg, logits, row_stride, rows, a.z);
    if (st != AED_OK || rows == 0) return st;
    if ((st = check_words("uniforms, tokens, logp, temperatures, top_ks, top_ps, min_ps", {uniforms, tokens, logp, how->temperatures, how->top_ks, how->top_ps, how->min_ps}, 3)) != AED_OK)
        return st;
    a.uniforms = uniforms;
    a.temperature = how->temperature;
    a.top_k = how->top_k;
    a.top_p = how->top_p;
    a.min_p = how->min_p;
    a.temperatures = how->temperatures;
    a.top_ks = how->top_ks;
    a.top_ps = how->top_ps;
    a.min_ps = how->min_ps;
    a.tokens = tokens;
    a.logp = logp;
    int width = 0;  // a row's weights, 1 at most each, add up to less than 2^63
    while (((int64_t)1 << width) < p->cfg.vocab) ++width;
    a.weight_bits = width < 12 ? 50 : 62 - width;
    return hip_status(aed::launch_sample(a, p->cfg.dtype == 1, p->stream), "aed_sample");
}

aed_status aed_top_create(const aed_top_config* cfg, void* hip_stream, aed_top** out) {
    if (out) *out = nullptr;
    aed_status st = check_config(cfg, out);
    if (st == AED_OK) st = check_list(cfg);
    if (st == AED_OK && cfg->top > cfg->vocab) return fail(AED_EINVAL, "top %d is above vocab %d", cfg->top, cfg->vocab);
    return st == AED_OK ? create(cfg, hip_stream, out) : st;
}
aed_status aed_top_destroy(aed_top* plan) { return finish(plan); }

aed_status aed_top_logits(aed_top* p, const void* logits, int64_t row_stride, int32_t rows, float* values, int32_t* ids, float* rest) {
    if (!p) return fail(AED_EINVAL, "plan is NULL");
    aed::TopArgs a = {};
    aed_status st = to_rows(p->cfg, logits, row_stride, rows, a.z);
    if (st != AED_OK || rows == 0) return st;
    if ((st = check_words("values, ids, rest", {values, ids, rest}, 3)) != AED_OK) return st;
    a.values = values;
    a.ids = ids;
    a.rest = rest;
    a.top = p->cfg.top;
    a.temperature = p->cfg.temperature;
    a.scale = (float)(kLog2e / (double)p->cfg.temperature);
    return hip_status(aed::launch_top(a, p->cfg.dtype == 1, p->stream), "aed_top_logits");
}

aed_status aed_distill_create(const aed_distill_config* cfg, void* hip_stream, aed_distill** out) {
    if (out) *out = nullptr;
    aed_status st = check_config(cfg, out);
    if (st == AED_OK) st = check_list(cfg);
    return st == AED_OK ? create(cfg, hip_stream, out) : st;
}
aed_status aed_distill_destroy(aed_distill* plan) { return finish(plan); }

aed_status aed_distill_forward(aed_distill* p, const void* logits, int64_t row_stride, int32_t rows, const float* values, const int32_t* ids, const float* rest,
                               const float* weights, float* loss, float* row_loss, float* stats) {
    if (!p || !loss) return fail(AED_EINVAL, "plan / loss is NULL");
    aed::DistillArgs a = {};
    aed_status st = to_rows(p->cfg, logits, row_stride, rows, a.z);
    if (st != AED_OK) return st;
    if ((st = check_words("values, ids, row_loss, stats, loss, rest, weights", {values, ids, row_loss, stats, loss, rest, weights}, rows > 0 ? 4 : 0)) != AED_OK) return st;
    a.values = values;
    a.ids = ids;
    a.rest = rest;
    a.weights = weights;
    a.loss = loss;
    a.row_loss = row_loss;
    a.stats = stats;
    set_temperature(p->cfg, a);
    return hip_status(aed::launch_distill_forward(a, p->cfg.dtype == 1, p->stream), "aed_distill_forward");
}

aed_status aed_distill_backward(aed_distill* p, const void* logits, int64_t row_stride, int32_t rows, const int32_t* ids, const float* weights, const float* stats,
                                const float* d_loss, void* d_logits, int64_t d_row_stride) {
    if (!p) return fail(AED_EINVAL, "plan is NULL");
    aed::DistillArgs a = {};
    aed_status st = to_rows(p->cfg, logits, row_stride, rows, a.z);
    if (st != AED_OK || rows == 0) return st;
    if ((st = check_words("ids, stats, weights, d_loss", {ids, stats, weights, d_loss}, 2)) != AED_OK) return st;
    if ((st = check_rows(d_logits, "d_logits", d_row_stride, rows, p->cfg.vocab, p->cfg.dtype)) != AED_OK) return st;
    if (rows > 1 && d_logits == logits && d_row_stride != row_stride) return fail(AED_EINVAL, "gradients in the logits' place need their row stride");
    a.ids = ids;
    a.weights = weights;
    a.stats = const_cast<float*>(stats);
    a.d_loss = d_loss;
    a.d_logits = d_logits;
    a.d_stride = rows > 1 ? d_row_stride : 0;
    set_temperature(p->cfg, a);
    return hip_status(aed::launch_distill_backward(a, p->cfg.dtype == 1, p->stream), "aed_distill_backward");
}

}  // extern "C"
