// attn.hip -- the packed attention's plan (work items for a batch's lengths) and C ABI.
//
// A plan cuts a batch's work into items (attn_plan.h), copies their lists to the device
// once, and serves every layer and both passes over the batch.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

#include "attn.h"

using namespace sieve;

struct sieve_attn {
  int device = 0;
  int32_t dtype = 0, heads = 0, kv_heads = 0, d = 0, dp = 0, causal = 0;
  int32_t nb = 0, distance = 0, span = 0;
  float scale = 0.f;
  int64_t queries = 0, keys = 0;
  bool few = false;          // forward tiles are of kAttnFewRows rows
  int32_t row_tiles = 0;     // dq tiles of one key head
  int32_t parts = 0;         // partial results of the forward pass
  int32_t kv_parts = 0;      // partial results of dk and dv
  int32_t nfwd = 0, ndq = 0, ndkv = 0, njoins = 0, nkv_joins = 0;
  void* mem = nullptr;       // everything below
  const AttnItem *fwd = nullptr, *dq = nullptr, *dkv = nullptr;
  const AttnJoin *joins = nullptr, *kv_joins = nullptr;
  const int16_t *bucket_of = nullptr, *range = nullptr;
};

namespace {

int64_t round256(int64_t n) { return (n + 255) & ~int64_t(255); }

int check_desc(const sieve_attn_desc& c) {
  if (!enc_dtype_ok(c.dtype))
    return set_error(SIEVE_EINVAL, "dtype = %d is not one of SIEVE_F32, SIEVE_F16, SIEVE_BF16",
                     c.dtype);
  if (c.heads < 1 || c.kv_heads < 1 || c.heads % c.kv_heads)
    return set_error(SIEVE_EINVAL, "heads = %d must be a multiple of kv_heads = %d", c.heads,
                     c.kv_heads);
  if (c.heads > 32768) return set_error(SIEVE_EUNSUPPORTED, "heads = %d is above 32768", c.heads);
  if (c.head_dim < 1) return set_error(SIEVE_EINVAL, "head_dim = %d must be >= 1", c.head_dim);
  if (c.head_dim > SIEVE_ATTN_MAX_DIM)
    return set_error(SIEVE_EUNSUPPORTED, "head_dim = %d is above %d", c.head_dim,
                     SIEVE_ATTN_MAX_DIM);
  if (c.causal != 0 && c.causal != 1) return set_error(SIEVE_EINVAL, "causal must be 0 or 1");
  if (!(c.scale > 0.f) || c.scale == INFINITY)
    return set_error(SIEVE_EINVAL, "scale must be > 0 and finite");
  if (c.num_buckets != 0) {
    if (c.num_buckets < 4 || c.num_buckets > 256 || c.num_buckets % 2)
      return set_error(SIEVE_EINVAL, "num_buckets = %d must be 0, or even and 4 .. 256",
                       c.num_buckets);
    const int side = c.causal ? c.num_buckets : c.num_buckets / 2;
    if (c.max_distance <= side / 2)
      return set_error(SIEVE_EINVAL, "max_distance = %d must be above %d, the exact buckets",
                       c.max_distance, side / 2);
    if ((int64_t)(c.heads / c.kv_heads) * (2 * (int64_t)c.max_distance + 2 * kAttnPad + 1) >
        SIEVE_ATTN_BIAS_SPAN)
      return set_error(SIEVE_EUNSUPPORTED,
                       "(heads / kv_heads) * (2 * max_distance + %d) is above %d",
                       2 * kAttnPad + 1, SIEVE_ATTN_BIAS_SPAN);
  }
  if (c.nseq < 0) return set_error(SIEVE_EINVAL, "nseq is negative");
  if (c.nseq > 0 && !c.q_offsets) return set_error(SIEVE_EINVAL, "q_offsets is NULL");
  const int64_t G = c.heads / c.kv_heads;
  for (int which = 0; which < 2; ++which) {
    const int64_t* o = which ? c.k_offsets : c.q_offsets;
    if (!o || c.nseq == 0) continue;
    const char* name = which ? "k_offsets" : "q_offsets";
    if (o[0] != 0) return set_error(SIEVE_EINVAL, "%s[0] must be 0", name);
    for (int64_t s = 0; s < c.nseq; ++s) {
      if (o[s + 1] < o[s])
        return set_error(SIEVE_EINVAL, "%s decreases at %lld", name, (long long)s);
      if (o[s + 1] - o[s] > kMaxRows / (which ? 1 : G))
        return set_error(SIEVE_EUNSUPPORTED, "sequence %lld of %s is too long", (long long)s,
                         name);
    }
    if (o[c.nseq] > kMaxTokens)
      return set_error(SIEVE_EUNSUPPORTED, "%s ends above %lld", name, (long long)kMaxTokens);
  }
  return SIEVE_OK;
}

int create(const sieve_attn_desc& c, hipStream_t stream, sieve_attn* p) {
  const int64_t *qo = c.q_offsets, *ko = c.k_offsets ? c.k_offsets : c.q_offsets;
  const int G = c.heads / c.kv_heads;
  p->dtype = c.dtype;
  p->heads = c.heads;
  p->kv_heads = c.kv_heads;
  p->d = c.head_dim;
  p->dp = c.head_dim <= 32 ? 32 : c.head_dim <= 64 ? 64 : c.head_dim <= 96 ? 96 : 128;
  p->causal = c.causal;
  p->scale = c.scale;
  p->queries = c.nseq ? qo[c.nseq] : 0;
  p->keys = c.nseq ? ko[c.nseq] : 0;
  AttnLists lists;
  if (!make_lists(qo, ko, c.nseq, c.kv_heads, G, c.causal != 0, &lists))
    return set_error(SIEVE_EUNSUPPORTED, "the batch has too many tiles");
  p->few = lists.few;
  p->row_tiles = lists.row_tiles;
  p->parts = lists.parts;
  p->kv_parts = lists.kv_parts;
  std::vector<int16_t> buckets, range;
  if (c.num_buckets) {
    p->nb = c.num_buckets;
    p->distance = c.max_distance;
    p->span = 2 * (c.max_distance + kAttnPad) + 1;
    range.assign(2 * p->nb, 0);
    for (int i = 0; i < p->span; ++i) {
      const int rel = std::clamp(i - c.max_distance - kAttnPad, -c.max_distance, c.max_distance);
      const int b = bucket_of(rel, c.num_buckets, c.max_distance, c.causal != 0);
      buckets.push_back((int16_t)b);
      if (range[2 * b + 1] == 0) range[2 * b] = (int16_t)i;
      range[2 * b + 1] = (int16_t)(i + 1);
    }
  }
  p->nfwd = (int32_t)lists.fwd.size();
  p->ndq = (int32_t)lists.dq.size();
  p->ndkv = (int32_t)lists.dkv.size();
  p->njoins = (int32_t)lists.joins.size();
  p->nkv_joins = (int32_t)lists.kv_joins.size();

  // one allocation, one copy
  std::vector<uint8_t> host;
  size_t at[7];
  auto add = [&](int i, const void* v, size_t bytes) {
    at[i] = host.size();
    host.resize(round256(host.size() + bytes));
    if (bytes) memcpy(host.data() + at[i], v, bytes);
  };
  add(0, lists.fwd.data(), lists.fwd.size() * sizeof(AttnItem));
  add(1, lists.dq.data(), lists.dq.size() * sizeof(AttnItem));
  add(2, lists.dkv.data(), lists.dkv.size() * sizeof(AttnItem));
  add(3, lists.joins.data(), lists.joins.size() * sizeof(AttnJoin));
  add(4, buckets.data(), buckets.size() * sizeof(int16_t));
  add(5, range.data(), range.size() * sizeof(int16_t));
  add(6, lists.kv_joins.data(), lists.kv_joins.size() * sizeof(AttnJoin));
  ENC_HIP_TRY(hipGetDevice(&p->device));
  if (host.empty()) return SIEVE_OK;
  ENC_HIP_TRY(hipMalloc(&p->mem, host.size()));
  ENC_HIP_TRY(hipMemcpyAsync(p->mem, host.data(), host.size(), hipMemcpyHostToDevice, stream));
  ENC_HIP_TRY(hipStreamSynchronize(stream));
  uint8_t* m = (uint8_t*)p->mem;
  p->fwd = (const AttnItem*)(m + at[0]);
  p->dq = (const AttnItem*)(m + at[1]);
  p->dkv = (const AttnItem*)(m + at[2]);
  p->joins = (const AttnJoin*)(m + at[3]);
  p->bucket_of = (const int16_t*)(m + at[4]);
  p->range = (const int16_t*)(m + at[5]);
  p->kv_joins = (const AttnJoin*)(m + at[6]);
  return SIEVE_OK;
}

// Workspace layouts.  Offsets in bytes.
struct FwdSpace {
  int64_t ml, bytes;
};
FwdSpace fwd_space(const sieve_attn* p) {
  const int64_t rows = (int64_t)p->parts * (p->few ? kAttnFewRows : kAttnRows);
  FwdSpace s;
  s.ml = round256(rows * p->dp * (int64_t)sizeof(float));
  s.bytes = p->parts ? s.ml + rows * kAttnStats * (int64_t)sizeof(float) : 0;
  return s;
}
struct BwdSpace {
  int64_t bias, most, kv, bytes;
};
BwdSpace bwd_space(const sieve_attn* p) {
  BwdSpace s;
  const int64_t tiles = (int64_t)p->row_tiles * p->kv_heads;
  s.bias = round256(p->queries * p->heads * (int64_t)sizeof(float));
  s.most = s.bias + round256(tiles * (p->heads / p->kv_heads) * p->nb * (int64_t)sizeof(float));
  s.kv = s.most + round256(p->dtype == SIEVE_F16 ? tiles * (int64_t)sizeof(float) : 0);
  s.bytes = s.kv + (int64_t)p->kv_parts * 2 * kAttnKeys * p->dp * (int64_t)sizeof(float);
  return s;
}

int check_heads(const sieve_heads* x, const char* name) {
  if (!x || !x->data) return set_error(SIEVE_EINVAL, "%s is NULL", name);
  if (x->token_stride < 0 || x->head_stride < 0)
    return set_error(SIEVE_EINVAL, "%s has a negative stride", name);
  return SIEVE_OK;
}
// Whether rows may be moved in 16-byte pieces at 32-bit offsets from a tile's first row.
bool heads_vec(const sieve_heads& x, int size, int G) {
  if ((((uintptr_t)x.data | (uint64_t)(x.token_stride * size) |
        (uint64_t)(x.head_stride * size)) & 15) != 0)
    return false;
  constexpr int64_t kMost = int64_t(1) << 40;  // far past 2^31: keeps the products small
  return std::min(x.token_stride, kMost) * kAttnRows * size +
             std::min(x.head_stride, kMost) * G * size + SIEVE_ATTN_MAX_DIM * size <
         (int64_t(1) << 31);
}

int check_plan(const sieve_attn* p) {
  if (!p) return set_error(SIEVE_EINVAL, "plan is NULL");
  int dev = 0;
  ENC_HIP_TRY(hipGetDevice(&dev));
  if (dev != p->device) return set_error(SIEVE_EINVAL, "current device differs from the plan's");
  return SIEVE_OK;
}
int check_workspace(int64_t need, const void* w, int64_t bytes) {
  if (need > 0 && (!w || bytes < need || ((uintptr_t)w & 15)))
    return set_error(SIEVE_EINVAL, "workspace must be 16-byte aligned and hold %lld bytes",
                     (long long)need);
  return SIEVE_OK;
}

AttnArgs common_args(const sieve_attn* p, const uint8_t* key_mask, const void* bias) {
  AttnArgs a{};
  a.key_mask = key_mask;
  a.bias = p->nb ? bias : nullptr;
  a.G = p->heads / p->kv_heads;
  while ((int64_t(1) << a.g_shift) < a.G) ++a.g_shift;
  a.g_mul = (uint32_t)(((uint64_t(1) << (31 + a.g_shift)) + a.G - 1) / a.G);
  a.heads = p->heads;
  a.d = p->d;
  a.causal = p->causal;
  a.scale = p->scale;
  a.nb = p->nb;
  a.distance = p->distance;
  a.span = p->span;
  a.bucket_of = p->bucket_of;
  a.range = p->range;
  a.row_tiles = p->row_tiles;
  return a;
}

hipError_t launch(const sieve_attn* p, AttnKind kind, const AttnArgs& a, int grid,
                  hipStream_t s) {
  switch (p->dtype) {
    case SIEVE_F32: return attn_launch_f32(kind, p->dp, a, grid, s);
    case SIEVE_F16: return attn_launch_f16(kind, p->dp, a, grid, s);
    default: return attn_launch_bf16(kind, p->dp, a, grid, s);
  }
}

}  // namespace

SIEVE_API int sieve_attn_create(const sieve_attn_desc* desc, void* stream, sieve_attn** out) {
  clear_error();
  if (!desc || !out) return set_error(SIEVE_EINVAL, "desc and out must be non-NULL");
  *out = nullptr;
  if (int st = check_desc(*desc)) return st;
  sieve_attn* p = new (std::nothrow) sieve_attn;
  if (!p) return set_error(SIEVE_ENOMEM, "host memory");
  int st;
  try {
    st = create(*desc, (hipStream_t)stream, p);
  } catch (const std::bad_alloc&) {
    st = set_error(SIEVE_ENOMEM, "host memory for the plan's work list");
  }
  if (st) {
    sieve_attn_free(p);
    return st;
  }
  *out = p;
  return SIEVE_OK;
}

SIEVE_API void sieve_attn_free(sieve_attn* plan) {
  if (!plan) return;
  if (plan->mem) (void)hipFree(plan->mem);
  delete plan;
}

SIEVE_API int64_t sieve_attn_workspace(const sieve_attn* plan, int32_t backward) {
  clear_error();
  if (!plan) return set_error(SIEVE_EINVAL, "plan is NULL");
  return backward ? bwd_space(plan).bytes : fwd_space(plan).bytes;
}

SIEVE_API int sieve_attn_forward(const sieve_attn* plan, const sieve_heads* q,
                                 const sieve_heads* k, const sieve_heads* v,
                                 const uint8_t* key_mask, const void* bias, const sieve_heads* o,
                                 float* lse, void* workspace, int64_t workspace_bytes,
                                 void* stream) {
  clear_error();
  if (!plan) return set_error(SIEVE_EINVAL, "plan is NULL");
  const sieve_attn* p = plan;
  if (p->queries == 0) return SIEVE_OK;
  int st;
  if ((st = check_heads(q, "q")) || (st = check_heads(o, "o"))) return st;
  if (p->keys > 0 && ((st = check_heads(k, "k")) || (st = check_heads(v, "v")))) return st;
  if (p->nb && !bias) return set_error(SIEVE_EINVAL, "bias is NULL and the plan has buckets");
  if (!p->nb && bias) return set_error(SIEVE_EINVAL, "bias given and the plan has no buckets");
  const FwdSpace sp = fwd_space(p);
  if ((st = check_workspace(sp.bytes, workspace, workspace_bytes))) return st;
  if ((st = check_plan(p))) return st;
  AttnArgs a = common_args(p, key_mask, bias);
  a.q = *q;
  a.o = *o;
  if (p->keys > 0) {
    a.k = *k;
    a.v = *v;
  }
  a.lse = lse;
  const int size = enc_size(p->dtype);
  a.vec = p->d * size % 16 == 0 && heads_vec(a.q, size, a.G) && heads_vec(a.o, size, a.G) &&
          heads_vec(a.k, size, 1) && heads_vec(a.v, size, 1);
  a.part_o = (float*)workspace;
  a.part_ml = (float*)((uint8_t*)workspace + sp.ml);
  a.items = p->fwd;
  a.joins = p->joins;
  a.nitems = p->nfwd;
  hipStream_t s = (hipStream_t)stream;
  ENC_HIP_TRY(launch(p, p->few ? kAttnFwdFew : kAttnFwd, a, p->nfwd, s));
  ENC_HIP_TRY(launch(p, p->few ? kAttnJoinFew : kAttnJoin, a, p->njoins, s));
  return SIEVE_OK;
}

SIEVE_API int sieve_attn_backward(const sieve_attn* plan, const sieve_heads* dout,
                                  const sieve_heads* q, const sieve_heads* k,
                                  const sieve_heads* v, const sieve_heads* o, const float* lse,
                                  const uint8_t* key_mask, const void* bias,
                                  const sieve_heads* dq, const sieve_heads* dk,
                                  const sieve_heads* dv, void* dbias, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  clear_error();
  if (!plan) return set_error(SIEVE_EINVAL, "plan is NULL");
  const sieve_attn* p = plan;
  int st;
  if (p->queries > 0) {
    if ((st = check_heads(dout, "dout")) || (st = check_heads(q, "q")) ||
        (st = check_heads(o, "o")) || (st = check_heads(dq, "dq")))
      return st;
    if (!lse) return set_error(SIEVE_EINVAL, "lse is NULL");
  }
  if (p->keys > 0 && ((st = check_heads(k, "k")) || (st = check_heads(v, "v")) ||
                      (st = check_heads(dk, "dk")) || (st = check_heads(dv, "dv"))))
    return st;
  if (p->nb && !bias) return set_error(SIEVE_EINVAL, "bias is NULL and the plan has buckets");
  if (!p->nb && (bias || dbias))
    return set_error(SIEVE_EINVAL, "bias or dbias given and the plan has no buckets");
  const BwdSpace sp = bwd_space(p);
  if ((st = check_workspace(sp.bytes, workspace, workspace_bytes))) return st;
  if ((st = check_plan(p))) return st;
  AttnArgs a = common_args(p, key_mask, bias);
  if (p->queries > 0) {
    a.dout = *dout;
    a.q = *q;
    a.o = *o;
    a.dq = *dq;
  }
  if (p->keys > 0) {
    a.k = *k;
    a.v = *v;
    a.dk = *dk;
    a.dv = *dv;
  }
  a.lse = const_cast<float*>(lse);
  a.dbias = dbias;
  const int size = enc_size(p->dtype);
  a.vec = p->d * size % 16 == 0;
  for (const sieve_heads* x : {&a.q, &a.o, &a.dout, &a.dq})
    a.vec = a.vec && heads_vec(*x, size, a.G);
  for (const sieve_heads* x : {&a.k, &a.v, &a.dk, &a.dv})
    a.vec = a.vec && heads_vec(*x, size, 1);
  uint8_t* w = (uint8_t*)workspace;
  a.dsum = (float*)w;
  a.part_bias = (float*)(w + sp.bias);
  a.part_max = (float*)(w + sp.most);
  a.part_kv = (float*)(w + sp.kv);
  hipStream_t s = (hipStream_t)stream;
  a.items = p->dq;
  a.nitems = p->ndq;
  ENC_HIP_TRY(launch(p, kAttnDq, a, p->ndq, s));
  a.items = p->dkv;
  a.nitems = p->ndkv;
  ENC_HIP_TRY(launch(p, kAttnDkv, a, p->ndkv + (dbias ? p->heads : 0), s));
  a.joins = p->kv_joins;
  ENC_HIP_TRY(launch(p, kAttnDkvJoin, a, p->nkv_joins, s));
  return SIEVE_OK;
}
