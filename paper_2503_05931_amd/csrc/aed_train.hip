// Host side of include/aed_train.h: argument checks, workspaces and launches of ragged attention and the preference loss.
#include "../../include/aed_train.h"

#include "attn_plan.h"
#include "attn_ragged.h"
#include "host_calls.h"
#include "preference.h"

static_assert(sizeof(aed::PlanItem) == sizeof(aed::RaggedItem) && sizeof(aed::PlanJoin) == sizeof(aed::RaggedJoin), "the lists are copied as they are");

thread_local char aed::train_error[512] = "";

namespace {

using aed::Arena;
using aed::fail;
using aed::finish;
using aed::guarded;
using aed::hip_status;
using aed::start;

constexpr int64_t kMost = 0x7fffffff;
constexpr int64_t kMostStart = (int64_t)1 << 38;  // times the bytes between rows (kAttnMaxPitch, 2^24 less a few): below 2^62
constexpr int64_t kMostStride = (int64_t)1 << 38;  // elements; in bytes and times the heads (2^16) below 2^57

}  // namespace

struct aed_attn {
    aed_attn_config cfg;
    hipStream_t stream = nullptr;
    aed::AttnPlan plan;
    Arena arena;
    size_t forward, joins, dq, dkv, zeros, bucket_of, bucket_range, part_o, part_ml, delta, large, part_bias;
    char* ws = nullptr;
    int64_t k_rows = 0;  // rows that the keys' tensors have: up to the last one that is read
    int span = 0;
};

namespace {

aed_status check_attn(const aed_attn_config* c, const int32_t* q_lens, const int32_t* k_lens, const int64_t* k_starts, int32_t batch) {
    if (!c || !q_lens || !k_lens) return fail(AED_EINVAL, "cfg / q_lens / k_lens is NULL");
    if (c->struct_size != sizeof(aed_attn_config)) return fail(AED_EINVAL, "struct_size %u, expected %zu", c->struct_size, sizeof(aed_attn_config));
    if (batch < 1) return fail(AED_EINVAL, "batch must be >= 1");
    if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads != 0)
        return fail(AED_EINVAL, "n_heads %d is no multiple of n_kv_heads %d", c->n_heads, c->n_kv_heads);
    if (c->dtype != 0 && c->dtype != 1) return fail(AED_EINVAL, "dtype must be 0 or 1");
    if ((c->causal | c->bias_bidirectional | c->training) & ~1) return fail(AED_EINVAL, "causal, bias_bidirectional and training are 0 or 1");
    if (!(c->scale >= 0.f) || !std::isfinite(c->scale)) return fail(AED_EINVAL, "scale must be a finite number >= 0");
    if (c->bias_buckets < 0) return fail(AED_EINVAL, "bias_buckets must be >= 0");
    if (c->bias_buckets > 0) {
        if (c->bias_bidirectional && c->bias_buckets % 2 != 0) return fail(AED_EINVAL, "a bidirectional bias needs an even number of buckets");
        const int side = c->bias_bidirectional ? c->bias_buckets / 2 : c->bias_buckets;
        if (side < 2) return fail(AED_EINVAL, "bias_buckets %d: a side has at least 2 buckets", c->bias_buckets);
        if (c->bias_max_distance <= side / 2) return fail(AED_EINVAL, "bias_max_distance %d must be above %d", c->bias_max_distance, side / 2);
        if (c->bias_buckets > 256) return fail(AED_EUNSUPPORTED, "more than 256 bias buckets");
        if (c->bias_max_distance > 1024) return fail(AED_EUNSUPPORTED, "bias_max_distance above 1024");
    }
    if (c->training && k_starts) return fail(AED_EINVAL, "training needs packed keys (k_starts NULL)");
    int64_t q_rows = 0, k_rows = 0;
    for (int b = 0; b < batch; ++b) {
        if (q_lens[b] < 0) return fail(AED_EINVAL, "q_lens[%d] = %d", b, q_lens[b]);
        if (k_lens[b] < 0) return fail(AED_EINVAL, "k_lens[%d] = %d", b, k_lens[b]);
        if (k_starts && (k_starts[b] < 0 || k_starts[b] > kMostStart)) return fail(AED_EINVAL, "k_starts[%d] is negative or too large", b);
        q_rows += q_lens[b];
        k_rows += k_lens[b];
    }
    if (c->head_dim != 64 && c->head_dim != 128) return fail(AED_EUNSUPPORTED, "head_dim %d (64 and 128 have kernels)", c->head_dim);
    // positions and distances are 32-bit: a key's place less a row's stays in range below 2^30
    for (int b = 0; b < batch; ++b)
        if (q_lens[b] > (1 << 30) || k_lens[b] > (1 << 30)) return fail(AED_EUNSUPPORTED, "a length above 2^30");
    if (q_rows > kMost || k_rows > kMost) return fail(AED_EUNSUPPORTED, "more than 2^31 - 1 query rows or keys");
    if (c->n_heads > 65535) return fail(AED_EUNSUPPORTED, "more than 65535 heads");
    return AED_OK;
}

aed_status lay_out(aed_attn& p, const int32_t* q_lens, const int32_t* k_lens, const int64_t* k_starts, int32_t batch) {
    const aed_attn_config& c = p.cfg;
    p.plan = aed::plan_attention(q_lens, k_lens, k_starts, batch, c.n_heads, c.n_kv_heads, c.causal != 0, c.training != 0, aed::kAttnRows,
                                 c.dtype == 0 && c.head_dim == 128 ? 0 : aed::kAttnPair, aed::kAttnFew, c.dtype == 1, c.head_dim);  // wide rows have no pairs
    const int64_t reduce = c.training ? ((int64_t)c.bias_buckets * c.n_heads + 3) / 4 : 0;  // workgroups of the bias's gradient, in the launch of the keys'
    if (std::max(p.plan.forward_groups, std::max(p.plan.dq_groups, p.plan.dkv_groups + reduce)) > aed::kPlanGrid)
        return fail(AED_EUNSUPPORTED, "more than 2^24 - 1 workgroups in a launch");
    p.k_rows = 0;
    for (int b = 0; b < batch; ++b) {
        if (!k_starts) p.k_rows += k_lens[b];
        else if (k_lens[b] > 0) p.k_rows = std::max(p.k_rows, k_starts[b] + k_lens[b]);
    }
    p.forward = p.arena.table(p.plan.forward);
    p.joins = p.arena.table(p.plan.joins);
    p.dq = p.arena.table(p.plan.dq);
    p.dkv = p.arena.table(p.plan.dkv);
    p.zeros = p.arena.table(std::vector<char>(512, 0));
    std::vector<uint8_t> of;
    std::vector<int2> range(c.bias_buckets, int2{0, 0});
    if (c.bias_buckets > 0) of = aed::bucket_places(c.bias_buckets, c.bias_max_distance, c.bias_bidirectional != 0);
    p.span = (int)of.size();
    for (int i = p.span - 1; i >= 0; --i) {  // a bucket's places lie side by side
        int2& r = range[of[i]];
        if (r.y == 0) r.y = i + 1 + aed::kAttnMargin;
        r.x = i + aed::kAttnMargin;
    }
    if (p.span > 0) {  // what is beyond an end is the end's
        range[of.front()].x = 0;
        range[of.back()].y = p.span + 2 * aed::kAttnMargin;
    }
    p.bucket_of = p.arena.table(of);
    p.bucket_range = p.arena.table(range);
    const size_t part_rows = (size_t)p.plan.n_parts * c.n_heads * p.plan.tile_rows;
    p.part_o = p.arena.scratch(part_rows * c.head_dim * sizeof(float));
    p.part_ml = p.arena.scratch(part_rows * sizeof(float2));
    p.delta = p.arena.scratch(c.training ? (size_t)p.plan.q_rows * c.n_heads * sizeof(float) : 0);
    p.large = p.arena.scratch(c.training && c.bias_buckets ? (size_t)p.plan.q_rows * c.n_heads * sizeof(float2) : 0);
    p.part_bias = p.arena.scratch(c.training ? p.plan.dq.size() * c.n_heads * c.bias_buckets * sizeof(float) : 0);
    return AED_OK;
}

// rows: how many the tensor has
aed_status to_tensor(const aed_rows* t, const char* name, int64_t rows, int heads, int head_dim, int es, bool output, aed::AttnTensor& to) {
    if (rows == 0) {
        to = aed::AttnTensor{nullptr, 0, 0};
        return AED_OK;
    }
    if (!t || !t->data) return fail(AED_EINVAL, "%s is NULL", name);
    if ((uintptr_t)t->data % 16 != 0) return fail(AED_EINVAL, "%s is not aligned to 16 bytes", name);
    const int64_t strides[2] = {rows > 1 ? t->row_stride : 0, heads > 1 ? t->head_stride : 0};
    for (int i = 0; i < 2; ++i) {
        if (strides[i] < 0 || strides[i] > kMostStride) return fail(AED_EINVAL, "%s: a stride is negative or above 2^38", name);
        if (strides[i] * es % 16 != 0) return fail(AED_EINVAL, "%s: a stride of %lld elements is no multiple of 16 bytes", name, (long long)strides[i]);
    }
    if (strides[0] > aed::kAttnMaxPitch / es) return fail(AED_EUNSUPPORTED, "%s: more than %d bytes between rows", name, aed::kAttnMaxPitch);
    if (output && aed::vectors_overlap(rows, strides[0], heads, strides[1], head_dim)) return fail(AED_EINVAL, "%s: rows or heads of an output overlap", name);
    to = aed::AttnTensor{static_cast<char*>(t->data), strides[0] * es, strides[1] * es};
    return AED_OK;
}

aed_status common_args(const aed_attn* p, const aed_rows* q, const aed_rows* k, const aed_rows* v, const void* bias, const uint8_t* key_mask,
                       const aed_rows* out, const float* lse, bool writes_out, aed::RaggedArgs& a) {
    const aed_attn_config& c = p->cfg;
    const int es = c.dtype == 1 ? 2 : 4;
    aed_status st;
    if ((st = to_tensor(q, "q", p->plan.q_rows, c.n_heads, c.head_dim, es, false, a.q)) != AED_OK) return st;
    if ((st = to_tensor(k, "k", p->k_rows, c.n_kv_heads, c.head_dim, es, false, a.k)) != AED_OK) return st;
    if ((st = to_tensor(v, "v", p->k_rows, c.n_kv_heads, c.head_dim, es, false, a.v)) != AED_OK) return st;
    if ((st = to_tensor(out, "out", p->plan.q_rows, c.n_heads, c.head_dim, es, writes_out, a.o)) != AED_OK) return st;
    if (p->plan.q_rows > 0 && !lse) return fail(AED_EINVAL, "lse is NULL");
    if ((uintptr_t)lse % 4 != 0) return fail(AED_EINVAL, "lse is not aligned to 4 bytes");
    if ((c.bias_buckets > 0) != (bias != nullptr)) return fail(AED_EINVAL, c.bias_buckets > 0 ? "bias is NULL" : "the handle was made without a bias");
    if ((uintptr_t)bias % es != 0) return fail(AED_EINVAL, "bias is not aligned to its elements");
    a.lse = const_cast<float*>(lse);
    a.key_mask = key_mask;
    a.bias = bias;
    a.zeros = p->ws + p->zeros;
    a.bucket_of = reinterpret_cast<const uint8_t*>(p->ws + p->bucket_of);
    a.bucket_range = reinterpret_cast<const int2*>(p->ws + p->bucket_range);
    a.delta = reinterpret_cast<float*>(p->ws + p->delta);
    a.large = reinterpret_cast<float2*>(p->ws + p->large);
    a.part_o = reinterpret_cast<float*>(p->ws + p->part_o);
    a.part_ml = reinterpret_cast<float2*>(p->ws + p->part_ml);
    a.part_bias = reinterpret_cast<float*>(p->ws + p->part_bias);
    a.joins = reinterpret_cast<const aed::RaggedJoin*>(p->ws + p->joins);
    a.scale = c.scale > 0.f ? c.scale : 1.f / sqrtf((float)c.head_dim);
    a.heads = c.n_heads;
    a.share = c.n_heads / c.n_kv_heads;
    a.causal = c.causal;
    a.buckets = c.bias_buckets;
    a.max_distance = c.bias_max_distance;
    a.span = p->span;
    return AED_OK;
}
const aed::RaggedItem* items(const aed_attn* p, size_t at) { return reinterpret_cast<const aed::RaggedItem*>(p->ws + at); }

}  // namespace

struct aed_preference {
    aed_preference_config cfg;
    hipStream_t stream = nullptr;
    Arena arena;
    size_t seq_of, seq_start, arrived, gain;
    char* ws = nullptr;
    int rows = 0, pairs = 0;
};

namespace {

aed_status check_preference(const aed_preference_config* c, const int32_t* seq_lens, int32_t n_pairs) {
    if (!c || !seq_lens) return fail(AED_EINVAL, "cfg / seq_lens is NULL");
    if (c->struct_size != sizeof(aed_preference_config)) return fail(AED_EINVAL, "struct_size %u, expected %zu", c->struct_size, sizeof(aed_preference_config));
    if (n_pairs < 1) return fail(AED_EINVAL, "n_pairs must be >= 1");
    if (n_pairs > kMost / 4) return fail(AED_EUNSUPPORTED, "too many pairs");
    if (c->vocab < 1) return fail(AED_EINVAL, "vocab must be >= 1");
    if (c->dtype != 0 && c->dtype != 1) return fail(AED_EINVAL, "dtype must be 0 or 1");
    if (!(c->beta > 0.f) || !std::isfinite(c->beta)) return fail(AED_EINVAL, "beta must be a finite number > 0");
    if (!(c->label_smoothing >= 0.f && c->label_smoothing < 0.5f)) return fail(AED_EINVAL, "label_smoothing must be in [0, 0.5)");
    int64_t rows = 0;
    for (int i = 0; i < 2 * n_pairs; ++i) {
        if (seq_lens[i] < 0) return fail(AED_EINVAL, "seq_lens[%d] = %d", i, seq_lens[i]);
        rows += seq_lens[i];
    }
    if (rows > 4 * aed::kPlanGrid) return fail(AED_EUNSUPPORTED, "more than 2^26 - 4 rows");  // four to a workgroup
    return AED_OK;
}

void lay_out(aed_preference& p, const int32_t* seq_lens, int32_t n_pairs) {
    std::vector<int32_t> of, start(1, 0);
    for (int i = 0; i < 2 * n_pairs; ++i) {
        of.insert(of.end(), (size_t)seq_lens[i], i);
        start.push_back((int32_t)of.size());
    }
    p.rows = (int)of.size();
    p.pairs = n_pairs;
    p.seq_of = p.arena.table(of);
    p.seq_start = p.arena.table(start);
    p.arrived = p.arena.table(std::vector<int32_t>(1, 0));
    p.gain = p.arena.scratch((size_t)p.rows * sizeof(float));
}

aed_status preference_args(const aed_preference* p, const void* logits, int64_t row_stride, const int32_t* labels, const float* ratio, const float* lse,
                           aed::PreferenceArgs& a) {
    const int es = p->cfg.dtype == 1 ? 2 : 4;
    if (!ratio) return fail(AED_EINVAL, "ratio is NULL");
    if (p->rows > 0) {
        if (!logits || !labels || !lse) return fail(AED_EINVAL, "logits / labels / lse is NULL");
        if ((uintptr_t)logits % es != 0) return fail(AED_EINVAL, "logits are not aligned to their elements");
        if (row_stride < p->cfg.vocab) return fail(AED_EINVAL, "row_stride %lld < vocab %d", (long long)row_stride, p->cfg.vocab);
    }
    if (((uintptr_t)labels | (uintptr_t)ratio | (uintptr_t)lse) % 4 != 0) return fail(AED_EINVAL, "labels, ratio or lse is not aligned to 4 bytes");
    if ((uintptr_t)lse % 8 != 0) return fail(AED_EINVAL, "lse is not aligned to its pairs of 8 bytes");
    a.logits = logits;
    a.row_stride = row_stride;
    a.labels = labels;
    a.ratio = const_cast<float*>(ratio);
    a.lse = reinterpret_cast<float2*>(const_cast<float*>(lse));
    a.gain = reinterpret_cast<float*>(p->ws + p->gain);
    a.arrived = reinterpret_cast<int32_t*>(p->ws + p->arrived);
    a.seq_of = reinterpret_cast<const int32_t*>(p->ws + p->seq_of);
    a.seq_start = reinterpret_cast<const int32_t*>(p->ws + p->seq_start);
    a.rows = p->rows;
    a.pairs = p->pairs;
    a.vocab = p->cfg.vocab;
    a.beta = p->cfg.beta;
    a.smoothing = p->cfg.label_smoothing;
    return AED_OK;
}

}  // namespace

extern "C" {

const char* aed_train_last_error(void) { return aed::train_error; }

aed_status aed_attn_workspace_bytes(const aed_attn_config* cfg, const int32_t* q_lens, const int32_t* k_lens, const int64_t* k_starts, int32_t batch,
                                    size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(AED_EINVAL, "bytes is NULL");
        aed_status st = check_attn(cfg, q_lens, k_lens, k_starts, batch);
        if (st != AED_OK) return st;
        aed_attn p;
        p.cfg = *cfg;
        if ((st = lay_out(p, q_lens, k_lens, k_starts, batch)) != AED_OK) return st;
        *bytes = p.arena.total;
        return AED_OK;
    });
}

aed_status aed_attn_create(const aed_attn_config* cfg, const int32_t* q_lens, const int32_t* k_lens, const int64_t* k_starts, int32_t batch,
                           void* workspace, size_t workspace_bytes, void* hip_stream, aed_attn** out) {
    return guarded([&] {
        if (!out) return fail(AED_EINVAL, "out is NULL");
        *out = nullptr;
        aed_status st = check_attn(cfg, q_lens, k_lens, k_starts, batch);
        if (st != AED_OK) return st;
        aed_attn* p = new aed_attn;
        try {
            p->cfg = *cfg;
            st = lay_out(*p, q_lens, k_lens, k_starts, batch);
        } catch (...) {
            delete p;
            throw;
        }
        if (st != AED_OK) {
            delete p;
            return st;
        }
        return start(p, workspace, workspace_bytes, hip_stream, out);
    });
}

aed_status aed_attn_destroy(aed_attn* plan) { return finish(plan); }

aed_status aed_attn_forward(aed_attn* p, const aed_rows* q, const aed_rows* k, const aed_rows* v, const void* bias, const uint8_t* key_mask,
                            const aed_rows* out, float* lse) {
    if (!p) return fail(AED_EINVAL, "plan is NULL");
    aed::RaggedArgs a = {};
    const aed_status st = common_args(p, q, k, v, bias, key_mask, out, lse, true, a);
    if (st != AED_OK) return st;
    const bool bf16 = p->cfg.dtype == 1;
    a.items = items(p, p->forward);
    a.n_items = (int)p->plan.forward.size();
    hipError_t e = aed::launch_attn_forward(a, p->cfg.head_dim, bf16, p->plan.tile_rows, p->stream);
    if (e == hipSuccess) e = aed::launch_attn_join(a, p->cfg.head_dim, bf16, p->plan.tile_rows, (int)p->plan.joins.size(), p->stream);
    return hip_status(e, "aed_attn_forward");
}

aed_status aed_attn_backward(aed_attn* p, const aed_rows* d_out, const aed_rows* q, const aed_rows* k, const aed_rows* v, const aed_rows* out,
                             const float* lse, const void* bias, const uint8_t* key_mask, const aed_rows* dq, const aed_rows* dk,
                             const aed_rows* dv, void* d_bias) {
    if (!p) return fail(AED_EINVAL, "plan is NULL");
    const aed_attn_config& c = p->cfg;
    if (!c.training) return fail(AED_ESTATE, "the handle was not made for training");
    aed::RaggedArgs a = {};
    aed_status st = common_args(p, q, k, v, bias, key_mask, out, lse, false, a);
    if (st != AED_OK) return st;
    const bool bf16 = c.dtype == 1;
    const int es = bf16 ? 2 : 4;
    if ((st = to_tensor(d_out, "d_out", p->plan.q_rows, c.n_heads, c.head_dim, es, false, a.d_o)) != AED_OK) return st;
    if ((st = to_tensor(dq, "dq", p->plan.q_rows, c.n_heads, c.head_dim, es, true, a.dq)) != AED_OK) return st;
    if ((st = to_tensor(dk, "dk", p->k_rows, c.n_kv_heads, c.head_dim, es, true, a.dk)) != AED_OK) return st;
    if ((st = to_tensor(dv, "dv", p->k_rows, c.n_kv_heads, c.head_dim, es, true, a.dv)) != AED_OK) return st;
    if ((bias != nullptr) != (d_bias != nullptr)) return fail(AED_EINVAL, bias ? "d_bias is NULL" : "the handle was made without a bias");
    if ((uintptr_t)d_bias % es != 0) return fail(AED_EINVAL, "d_bias is not aligned to its elements");
    a.items = items(p, p->dq);
    a.n_items = a.bias_items = (int)p->plan.dq.size();
    a.d_bias = d_bias;
    hipError_t e = aed::launch_attn_dq(a, c.head_dim, bf16, p->plan.dq_rows, p->stream);
    a.items = items(p, p->dkv);
    a.n_items = (int)p->plan.dkv.size();
    if (e == hipSuccess) e = aed::launch_attn_dkv(a, c.head_dim, bf16, p->plan.dkv_keys, p->stream);
    return hip_status(e, "aed_attn_backward");
}

aed_status aed_preference_workspace_bytes(const aed_preference_config* cfg, const int32_t* seq_lens, int32_t n_pairs, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(AED_EINVAL, "bytes is NULL");
        const aed_status st = check_preference(cfg, seq_lens, n_pairs);
        if (st != AED_OK) return st;
        aed_preference p;
        lay_out(p, seq_lens, n_pairs);
        *bytes = p.arena.total;
        return AED_OK;
    });
}

aed_status aed_preference_create(const aed_preference_config* cfg, const int32_t* seq_lens, int32_t n_pairs, void* workspace, size_t workspace_bytes,
                                 void* hip_stream, aed_preference** out) {
    return guarded([&] {
        if (!out) return fail(AED_EINVAL, "out is NULL");
        *out = nullptr;
        const aed_status st = check_preference(cfg, seq_lens, n_pairs);
        if (st != AED_OK) return st;
        aed_preference* p = new aed_preference;
        try {
            p->cfg = *cfg;
            lay_out(*p, seq_lens, n_pairs);
        } catch (...) {
            delete p;
            throw;
        }
        return start(p, workspace, workspace_bytes, hip_stream, out);
    });
}

aed_status aed_preference_destroy(aed_preference* plan) { return finish(plan); }

aed_status aed_preference_forward(aed_preference* p, const void* logits, int64_t row_stride, const int32_t* labels, const float* ref_logp, float* loss,
                                  float* ratio, float* lse) {
    if (!p) return fail(AED_EINVAL, "plan is NULL");
    aed::PreferenceArgs a = {};
    const aed_status st = preference_args(p, logits, row_stride, labels, ratio, lse, a);
    if (st != AED_OK) return st;
    if (!loss || (p->rows > 0 && !ref_logp)) return fail(AED_EINVAL, "loss / ref_logp is NULL");
    if (((uintptr_t)loss | (uintptr_t)ref_logp) % 4 != 0) return fail(AED_EINVAL, "loss or ref_logp is not aligned to 4 bytes");
    a.loss = loss;
    a.ref = ref_logp;
    return hip_status(aed::launch_preference_forward(a, p->cfg.dtype == 1, p->stream), "aed_preference_forward");
}

aed_status aed_preference_backward(aed_preference* p, const void* logits, int64_t row_stride, const int32_t* labels, const float* ratio, const float* lse,
                                   const float* d_loss, void* d_logits, int64_t d_row_stride) {
    if (!p) return fail(AED_EINVAL, "plan is NULL");
    aed::PreferenceArgs a = {};
    const aed_status st = preference_args(p, logits, row_stride, labels, ratio, lse, a);
    if (st != AED_OK) return st;
    const int es = p->cfg.dtype == 1 ? 2 : 4;
    if (p->rows > 0) {
        if (!d_logits) return fail(AED_EINVAL, "d_logits is NULL");
        if ((uintptr_t)d_logits % es != 0) return fail(AED_EINVAL, "d_logits are not aligned to their elements");
        if (d_row_stride < p->cfg.vocab) return fail(AED_EINVAL, "d_row_stride %lld < vocab %d", (long long)d_row_stride, p->cfg.vocab);
        if (d_logits == logits && d_row_stride != row_stride) return fail(AED_EINVAL, "gradients in the logits' place need their row stride");
    }
    if ((uintptr_t)d_loss % 4 != 0) return fail(AED_EINVAL, "d_loss is not aligned to 4 bytes");
    a.d_loss = d_loss;
    a.d_logits = d_logits;
    a.d_row_stride = d_row_stride;
    return hip_status(aed::launch_preference_backward(a, p->cfg.dtype == 1, p->stream), "aed_preference_backward");
}

}  // extern "C"
