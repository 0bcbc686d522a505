// Entry points of the serving operators (included by ssd_api.cpp, whose error
// and pointer helpers they use): argument checks and launches, no state.
#pragma once

namespace {

// The array arguments of one call: each `bytes` of device memory of the current device, whole inside one
// allocation and aligned to its elements.  Asking the runtime takes 0.4 us an array, as long as a third of a small
// kernel's launch: an array in an allocation that an earlier one of the same call lies in is not asked for again
// (small tensors of a caching allocator share one).
struct ArrayCheck {
  int dev = -1, n = 0;
  const char* bad = nullptr;
  struct {
    uintptr_t base;
    size_t size;
  } seen[4];
  explicit ArrayCheck(void* stream) {
    hipDevice_t sd = -1;
    (void)hipGetLastError();  // what an earlier call of the thread left is not this one's (launched() asks for its own)
    if (hipGetDevice(&dev) != hipSuccess) {
      (void)hipGetLastError();
      bad = "no GPU";
    } else if (stream) {
      if (hipStreamGetDevice((hipStream_t)stream, &sd) != hipSuccess) {
        (void)hipGetLastError();
        bad = "stream";
      } else if (sd != dev) {
        bad = "stream (of another device)";
      }
    }
  }
  void need(const char* name, const void* p, size_t bytes, size_t align) {
    const uintptr_t at = (uintptr_t)p;
    if (bytes > (size_t)PTRDIFF_MAX) bad = name;  // (on any machine: no array is that long)
    if (bad || !bytes) return;
    if (!p || (at & (align - 1))) {
      bad = name;
      return;
    }
    for (int i = 0; i < n; ++i)
      if (at >= seen[i].base && at - seen[i].base < seen[i].size && bytes <= seen[i].size - (at - seen[i].base)) return;
    hipPointerAttribute_t attr;
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipPointerGetAttributes(&attr, p) != hipSuccess || attr.type != hipMemoryTypeDevice || attr.device != dev ||
        hipMemGetAddressRange(&base, &size, const_cast<void*>(p)) != hipSuccess) {
      (void)hipGetLastError();
      bad = name;
      return;
    }
    const size_t off = at - (uintptr_t)base;
    if (off > size || bytes > size - off) {
      bad = name;
      return;
    }
    if (n < 4) {
      seen[n].base = (uintptr_t)base;
      seen[n++].size = size;
    }
  }
  ssd_status status() const {
    return bad ? fail(SSD_E_INVAL, "%s: needs an aligned array of the current device, whole inside one allocation", bad)
               : SSD_OK;
  }
};

// bytes of rows of cols elements, ld apart; where they pass 64 bits, more than any array has
size_t span(size_t rows, size_t ld, size_t cols, size_t es) {
  size_t n = 0;
  if (!rows) return 0;
  return __builtin_mul_overflow(rows - 1, ld, &n) || __builtin_add_overflow(n, cols, &n) || __builtin_mul_overflow(n, es, &n)
             ? SIZE_MAX
             : n;
}

ssd_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SSD_OK : fail(SSD_E_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool block_ok(int T) { return T == 16 || T == 32 || T == 64 || T == 128; }

ssd_status check_cache(const ssd_kvq_cache* c) {
  if (!c) return fail(SSD_E_INVAL, "cache is NULL");
  if (!block_ok(c->block)) return fail(SSD_E_INVAL, "block = %d: 16, 32, 64 or 128 tokens", c->block);
  if (c->head_dim != 64 && c->head_dim != 128) return fail(SSD_E_INVAL, "head_dim = %d: 64 or 128", c->head_dim);
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535) return fail(SSD_E_INVAL, "n_kv_heads = %d", c->n_kv_heads);
  if (c->n_blocks < 1 || (int64_t)c->n_blocks * c->block > INT32_MAX)
    return fail(SSD_E_INVAL, "n_blocks = %d: n_blocks * block must lie in [1, 2^31)", c->n_blocks);
  return SSD_OK;
}

void need_cache(ArrayCheck& ck, const ssd_kvq_cache& c) {
  const size_t heads = (size_t)c.n_blocks * c.n_kv_heads, n = heads * c.block * c.head_dim;
  ck.need("cache k", c.k, n, 16);
  ck.need("cache v", c.v, n, 16);
  ck.need("cache k_exp", c.k_exp, heads, 1);
  ck.need("cache v_exp", c.v_exp, heads, 1);
}

bool dtype_ok(int dtype) { return dtype == SSD_F32 || dtype == SSD_BF16; }

// sizes only; a: everything of the launch but the arrays
ssd_status attn_sizes(const ssd_kvq_cache* c, const ssd_kvq_attn_params* p, KvqAttnArgs& a) {
  if (!p) return fail(SSD_E_INVAL, "params is NULL");
  const ssd_status cs = check_cache(c);
  if (cs != SSD_OK) return cs;
  if (!dtype_ok(p->dtype)) return fail(SSD_E_INVAL, "unknown dtype");
  if (p->n_seqs < 1 || p->n_rows < 1 || p->max_q < 1 || p->max_len < 1 || p->table_width < 1)
    return fail(SSD_E_INVAL, "n_seqs, n_rows, max_q, max_len and table_width must be positive");
  if (p->n_heads < 1 || p->n_heads % c->n_kv_heads || p->n_heads > 65535)
    return fail(SSD_E_INVAL, "n_heads = %d must be a multiple of n_kv_heads = %d", p->n_heads, c->n_kv_heads);
  if ((int64_t)p->n_seqs * p->max_q > INT32_MAX / p->n_heads)
    return fail(SSD_E_INVAL, "n_seqs * max_q * n_heads must stay below 2^31");
  const int64_t rows = (int64_t)p->max_q * (p->n_heads / c->n_kv_heads);
  if ((int64_t)p->n_seqs * c->n_kv_heads * ((rows + 15) / 16) >= 1 << 24)
    return fail(SSD_E_INVAL, "n_seqs * n_kv_heads * (max_q * query heads a KV head / 16, rounded up) must stay below 2^24");
  if ((int64_t)p->table_width * c->block > (1 << 30))
    return fail(SSD_E_INVAL, "table_width * block must be at most 2^30 positions");
  const int64_t cols = (int64_t)p->n_heads * c->head_dim;
  if (p->ld_q < cols || p->ld_out < cols) return fail(SSD_E_INVAL, "row lengths must be at least n_heads * head_dim");
  if (!std::isfinite(kvq_scale_log2(p->scale))) return fail(SSD_E_INVAL, "scale must be finite, below 2.3e38 in magnitude");
  a = KvqAttnArgs{};
  a.n_blocks = c->n_blocks;
  a.T = c->block;
  a.Hkv = c->n_kv_heads;
  a.D = c->head_dim;
  a.B = p->n_seqs;
  a.n_rows = p->n_rows;
  a.Hq = p->n_heads;
  a.max_q = p->max_q;
  a.max_len = (int)std::min<int64_t>(p->max_len, (int64_t)p->table_width * c->block);
  a.width = p->table_width;
  a.bf16 = p->dtype == SSD_BF16;
  a.ld_q = (size_t)p->ld_q;
  a.ld_o = (size_t)p->ld_out;
  a.scale = p->scale;
  return SSD_OK;
}

// settings and arrays of a sampling call of R rows (logits: checked where they are the caller's)
ssd_status sample_args(const ssd_sample_params& p, int R, const float* u, int32_t* tokens, float* probs, void* stream, SampleArgs& a,
                       const float* logits = nullptr) {
  if (!p.temperatures && (!std::isfinite(p.temperature) || p.temperature < 0.0))
    return fail(SSD_E_INVAL, "temperature must be a finite number >= 0");
  if ((!p.top_ps && std::isnan(p.top_p)) || (!p.min_ps && std::isnan(p.min_p)))
    return fail(SSD_E_INVAL, "top_p and min_p must be numbers");
  const size_t n = R;
  ArrayCheck ck(stream);
  if (logits) ck.need("logits", logits, span(n, p.ld, p.vocab, 4), 4);
  ck.need("u", u, n * 4, 4);
  ck.need("tokens", tokens, n * 4, 4);
  if (probs) ck.need("probs", probs, n * 4, 4);
  if (p.temperatures) ck.need("temperatures", p.temperatures, n * 4, 4);
  if (p.top_ks) ck.need("top_ks", p.top_ks, n * 4, 4);
  if (p.top_ps) ck.need("top_ps", p.top_ps, n * 4, 4);
  if (p.min_ps) ck.need("min_ps", p.min_ps, n * 4, 4);
  if (ck.bad) return ck.status();
  a = SampleArgs{R, p.vocab, p.top_k, 0, (size_t)p.ld, p.temperature, p.top_p, p.min_p, p.temperatures, p.top_ps, p.min_ps, p.top_ks,
                 logits, u, tokens, probs};
  return SSD_OK;
}

}  // namespace

extern "C" {

ssd_status ssd_kvq_slots(const ssd_kvq_slot_params* p, const int32_t* held, const int32_t* fresh, const int32_t* pool,
                         int32_t* table, int32_t* lens, int32_t* cu, int32_t* slots, int32_t* positions, int32_t* used,
                         void* stream) {
  g_err.clear();
  if (!p) return fail(SSD_E_INVAL, "params is NULL");
  if (!block_ok(p->block)) return fail(SSD_E_INVAL, "block = %d: 16, 32, 64 or 128 tokens", p->block);
  if (p->n_seqs < 1 || p->table_width < 1 || p->n_pool < 0 || p->n_rows < 0)
    return fail(SSD_E_INVAL, "n_seqs and table_width must be positive, n_pool and n_rows not negative");
  if (p->n_seqs > 1 << 20) return fail(SSD_E_INVAL, "n_seqs = %d: up to 2^20 requests", p->n_seqs);
  if (!held || !fresh || !table || !lens || !cu || !used || (p->n_pool && !pool) || (p->n_rows && (!slots || !positions)))
    return fail(SSD_E_INVAL, "NULL argument");
  const size_t B = p->n_seqs, n = p->n_rows;
  ArrayCheck ck(stream);
  ck.need("held", held, B * 4, 4);
  ck.need("fresh", fresh, B * 4, 4);
  ck.need("pool", pool, (size_t)p->n_pool * 4, 4);
  ck.need("table", table, B * p->table_width * 4, 4);
  ck.need("lens", lens, B * 4, 4);
  ck.need("cu", cu, (B + 1) * 4, 4);
  ck.need("slots", slots, n * 4, 4);
  ck.need("positions", positions, n * 4, 4);
  ck.need("used", used, 4, 4);
  if (ck.bad) return ck.status();
  kvq_slots(SlotArgs{p->n_seqs, p->block, p->table_width, p->n_pool, p->n_rows, held, fresh, pool, table, lens, cu, slots,
                     positions, used},
            (hipStream_t)stream);
  return launched("ssd_kvq_slots");
}

ssd_status ssd_rope_axes(const ssd_rope_params* p, int32_t T, const void* q, const void* k, const int32_t* positions,
                         void* q_out, void* k_out, void* stream) {
  g_err.clear();
  if (!p || !q || !k || !positions || !q_out || !k_out) return fail(SSD_E_INVAL, "NULL argument");
  if (T < 1 || T >= 1 << 25) return fail(SSD_E_INVAL, "T = %d outside [1, 2^25)", T);
  if (!dtype_ok(p->dtype)) return fail(SSD_E_INVAL, "unknown dtype");
  if (p->n_heads < 1 || p->n_kv_heads < 1 || p->n_heads > 65535 || p->n_kv_heads > 65535)
    return fail(SSD_E_INVAL, "n_heads and n_kv_heads must lie in [1, 65535]");
  if (p->head_dim < 2 || p->head_dim > 1024) return fail(SSD_E_INVAL, "head_dim = %d outside [2, 1024]", p->head_dim);
  if (p->n_axes < 1 || p->n_axes > SSD_ROPE_AXES) return fail(SSD_E_INVAL, "n_axes = %d outside [1, %d]", p->n_axes, SSD_ROPE_AXES);
  RopeArgs a{};
  int64_t half = 0;
  for (int i = 0; i < p->n_axes; ++i) {
    if (p->section[i] < 0) return fail(SSD_E_INVAL, "negative section");
    half += p->section[i];
    a.section[i] = p->section[i];
  }
  if (half < 1 || 2 * half > p->head_dim) return fail(SSD_E_INVAL, "sections sum to %lld pairs of head_dim = %d", (long long)half, p->head_dim);
  if (!std::isfinite(p->theta) || !(p->theta > 0.0)) return fail(SSD_E_INVAL, "theta must be a finite number > 0");
  const int64_t cq = (int64_t)p->n_heads * p->head_dim, ckv = (int64_t)p->n_kv_heads * p->head_dim;
  if (p->ld_q < cq || p->ld_q_out < cq || p->ld_k < ckv || p->ld_k_out < ckv)
    return fail(SSD_E_INVAL, "row lengths must be at least heads * head_dim");
  if ((q == q_out && p->ld_q != p->ld_q_out) || (k == k_out && p->ld_k != p->ld_k_out))
    return fail(SSD_E_INVAL, "an output in place of its input has the same row length");
  const size_t es = p->dtype == SSD_BF16 ? 2 : 4, t = T;
  ArrayCheck ck(stream);
  ck.need("q", q, span(t, p->ld_q, cq, es), es);
  ck.need("k", k, span(t, p->ld_k, ckv, es), es);
  ck.need("positions", positions, t * p->n_axes * 4, 4);
  ck.need("q_out", q_out, span(t, p->ld_q_out, cq, es), es);
  ck.need("k_out", k_out, span(t, p->ld_k_out, ckv, es), es);
  if (ck.bad) return ck.status();
  a.T = T;
  a.Hq = p->n_heads;
  a.Hkv = p->n_kv_heads;
  a.D = p->head_dim;
  a.half = (int)half;
  a.bf16 = p->dtype == SSD_BF16;
  a.log2_theta = std::log2(p->theta);
  a.ld_q = p->ld_q;
  a.ld_k = p->ld_k;
  a.ld_qo = p->ld_q_out;
  a.ld_ko = p->ld_k_out;
  a.q = q;
  a.k = k;
  a.qo = q_out;
  a.ko = k_out;
  a.pos = positions;
  rope_axes(a, (hipStream_t)stream);
  return launched("ssd_rope_axes");
}

ssd_status ssd_kvq_append(const ssd_kvq_cache* c, const ssd_kvq_append_params* p, const int32_t* slots, const void* k,
                          const void* v, void* stream) {
  g_err.clear();
  if (!p) return fail(SSD_E_INVAL, "params is NULL");
  const ssd_status cs = check_cache(c);
  if (cs != SSD_OK) return cs;
  if (!dtype_ok(p->dtype)) return fail(SSD_E_INVAL, "unknown dtype");
  if (p->n_rows < 0) return fail(SSD_E_INVAL, "n_rows = %d is negative", p->n_rows);
  const int64_t cols = (int64_t)c->n_kv_heads * c->head_dim;
  if (p->ld_k < cols || p->ld_v < cols) return fail(SSD_E_INVAL, "row lengths must be at least n_kv_heads * head_dim");
  if ((int64_t)(p->n_rows / kvq_append_window(p->n_rows) + 1) * c->n_kv_heads * 2 >= 1 << 24)
    return fail(SSD_E_INVAL, "n_rows = %d of %d heads: more than a launch takes", p->n_rows, c->n_kv_heads);
  if (p->n_rows == 0) return SSD_OK;
  if (!slots || !k || !v || !c->k || !c->v || !c->k_exp || !c->v_exp) return fail(SSD_E_INVAL, "NULL argument");
  const size_t es = p->dtype == SSD_BF16 ? 2 : 4, n = p->n_rows;
  ArrayCheck ck(stream);
  ck.need("slots", slots, n * 4, 4);
  ck.need("k", k, span(n, p->ld_k, cols, es), es);
  ck.need("v", v, span(n, p->ld_v, cols, es), es);
  need_cache(ck, *c);
  if (ck.bad) return ck.status();
  KvqAppendArgs a{(uint8_t*)c->k, (uint8_t*)c->v, c->k_exp, c->v_exp, c->n_blocks, c->block, c->n_kv_heads, c->head_dim,
                  p->n_rows, p->dtype == SSD_BF16, slots, k, v, (size_t)p->ld_k, (size_t)p->ld_v};
  kvq_append(a, (hipStream_t)stream);
  return launched("ssd_kvq_append");
}

int64_t ssd_kvq_workspace(const ssd_kvq_cache* c, const ssd_kvq_attn_params* p) {
  g_err.clear();
  KvqAttnArgs a;
  if (attn_sizes(c, p, a) != SSD_OK) return -1;
  return (int64_t)kvq_attn_workspace(a);
}

ssd_status ssd_kvq_attention(const ssd_kvq_cache* c, const ssd_kvq_attn_params* p, const void* q, const int32_t* cu,
                             const int32_t* lens, const int32_t* table, void* out, void* workspace, void* stream) {
  g_err.clear();
  KvqAttnArgs a;
  const ssd_status cs = attn_sizes(c, p, a);
  if (cs != SSD_OK) return cs;
  const size_t need = kvq_attn_workspace(a);
  if (!q || !cu || !lens || !table || !out || (need && !workspace) || !c->k || !c->v || !c->k_exp || !c->v_exp)
    return fail(SSD_E_INVAL, "NULL argument");
  if (p->workspace_bytes < (int64_t)need)
    return fail(SSD_E_INVAL, "workspace of %lld bytes: this call needs %zu", (long long)p->workspace_bytes, need);
  if (q == out && p->ld_q != p->ld_out) return fail(SSD_E_INVAL, "an output in place of its input has the same row length");
  const size_t es = p->dtype == SSD_BF16 ? 2 : 4, B = p->n_seqs;
  ArrayCheck ck(stream);
  ck.need("q", q, span(a.n_rows, a.ld_q, (size_t)a.Hq * a.D, es), es);
  ck.need("out", out, span(a.n_rows, a.ld_o, (size_t)a.Hq * a.D, es), es);
  ck.need("cu", cu, (B + 1) * 4, 4);
  ck.need("lens", lens, B * 4, 4);
  ck.need("table", table, B * a.width * 4, 4);
  ck.need("workspace", workspace, need, 16);
  need_cache(ck, *c);
  if (ck.bad) return ck.status();
  a.kc = (const uint8_t*)c->k;
  a.vc = (const uint8_t*)c->v;
  a.ke = c->k_exp;
  a.ve = c->v_exp;
  a.q = q;
  a.o = out;
  a.cu = cu;
  a.lens = lens;
  a.table = table;
  a.workspace = workspace;
  kvq_attention(a, (hipStream_t)stream);
  return launched("ssd_kvq_attention");
}

ssd_status ssd_sample_logits(const ssd_sample_params* p, int32_t R, const float* logits, const float* u, int32_t* tokens,
                             float* probs, void* stream) {
  g_err.clear();
  if (!p || !logits || !u || !tokens) return fail(SSD_E_INVAL, "NULL argument");
  if (R < 1 || R >= 1 << 22) return fail(SSD_E_INVAL, "R = %d outside [1, 2^22)", R);
  if (p->vocab < 1 || p->vocab > (1 << 18)) return fail(SSD_E_INVAL, "vocab = %d outside [1, 2^18]", p->vocab);
  if (p->ld < p->vocab) return fail(SSD_E_INVAL, "ld must be at least vocab");
  SampleArgs a;
  const ssd_status cs = sample_args(*p, R, u, tokens, probs, stream, a, logits);
  if (cs != SSD_OK) return cs;
  sample_logits(a, (hipStream_t)stream);
  return launched("ssd_sample_logits");
}

ssd_status ssd_session_sample(ssd_session* s, const ssd_sample_params* p, const float* u, int32_t* tokens, float* probs) {
  g_err.clear();
  if (!s || !p || !u || !tokens) return fail(SSD_E_INVAL, "NULL argument");
  if (s->poisoned) return fail(SSD_E_STATE, "session is poisoned");
  if (s->dm.Vimg > (1 << 18)) return fail(SSD_E_INVAL, "sampling takes up to 2^18 codes");
  SampleArgs a;
  const ssd_status cs = sample_args(*p, s->Bi, u, tokens, probs, s->stream, a);
  if (cs != SSD_OK) return cs;
  a.V = s->dm.Vimg;
  a.ld = (size_t)s->dm.Vimg;
  a.add = s->dm.img_lo;
  a.logits = s->carry;
  if (s->cfg) {
    cfg_mix(s->Bi, 0, s->dm.Vimg, s->cfg_w, nullptr, s->carry, nullptr, s->mcarry, s->stream);
    a.logits = s->mcarry;
  }
  sample_logits(a, s->stream);
  return launched("ssd_session_sample");
}

ssd_status ssd_session_set_axes(ssd_session* s, int32_t n_axes, const int32_t* section, const int32_t* positions) {
  g_err.clear();
  if (!s || !section || !positions) return fail(SSD_E_INVAL, "NULL argument");
  if (s->poisoned) return fail(SSD_E_STATE, "session is poisoned");
  if (n_axes < 1 || n_axes > SSD_ROPE_AXES) return fail(SSD_E_INVAL, "n_axes = %d outside [1, %d]", n_axes, SSD_ROPE_AXES);
  RopeTableArgs a{};
  int64_t half = 0;
  for (int i = 0; i < n_axes; ++i) {
    if (section[i] < 0) return fail(SSD_E_INVAL, "negative section");
    half += section[i];
    a.section[i] = section[i];
  }
  if (half != s->dm.D / 2) return fail(SSD_E_INVAL, "sections sum to %lld pairs, a head has %d", (long long)half, s->dm.D / 2);
  a.n = s->max_ctx - s->P;  // (at least one)
  for (int b = 0; b < s->B; ++b)
    if (s->f[b] != s->P) return fail(SSD_E_STATE, "positions behind the prompt are already committed");
  try {
    if (!s->axes) s->axes = s->mem.get<int>((size_t)SSD_ROPE_AXES * a.n);
  } catch (HipError& e) {
    return fail(SSD_E_OOM, "%s: %s", e.what, hipGetErrorString(e.e));
  }
  if (hipMemcpyAsync(s->axes, positions, (size_t)n_axes * a.n * 4, hipMemcpyDefault, s->stream) != hipSuccess) {
    (void)hipGetLastError();
    return fail(SSD_E_INVAL, "the positions could not be read");
  }
  if (!is_device_ptr(positions) && hipStreamSynchronize(s->stream) != hipSuccess) {  // the host's array may go at our return
    (void)hipGetLastError();
    return fail(SSD_E_DEVICE, "the positions' copy failed");
  }
  a.pos = s->axes;
  a.half = s->dm.D / 2;
  a.theta = (double)s->dm.theta;
  a.tab = s->rope + (size_t)s->P * a.half;
  (void)hipGetLastError();  // (as in ArrayCheck)
  rope_axes_table(a, s->stream);
  const ssd_status ls = launched("ssd_session_set_axes");
  if (ls != SSD_OK) s->poisoned = true;
  return ls;
}

ssd_status ssd_session_read_kv(ssd_session* s, int32_t layer, int32_t n, void* k_out, void* v_out) {
  g_err.clear();
  if (!s || !k_out || !v_out) return fail(SSD_E_INVAL, "NULL argument");
  if (s->poisoned) return fail(SSD_E_STATE, "session is poisoned");
  if (layer < 0 || layer >= s->dm.L) return fail(SSD_E_INVAL, "layer = %d of %d", layer, s->dm.L);
  for (int b = 0; b < s->B; ++b)
    if (n < 1 || n > s->f[b]) return fail(SSD_E_INVAL, "n = %d outside [1, frontier = %d]", n, s->f[b]);
  const size_t es = esize(s->dm), bytes = (size_t)s->B * n * s->dm.Hkv * s->dm.D * es;
  ArrayCheck ck(s->stream);
  ck.need("k_out", k_out, bytes, es);
  ck.need("v_out", v_out, bytes, es);
  if (ck.bad) return ck.status();
  const size_t at = (size_t)layer * s->kv_layer_elems * es;
  read_kv(s->dm, s->B, n, s->Lmax, (const char*)s->kc + at, (const char*)s->vc + at, k_out, v_out, s->stream);
  return launched("ssd_session_read_kv");
}

}  // extern "C"
