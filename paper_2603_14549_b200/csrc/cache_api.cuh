// Host side of the calls around the key / value cache (asap_rope, asap_cache_attention, asap_cache_evict, asap_cache_slot): checks of
// the arguments, scratch layout, launches.  Part of asap_api.cu.
#pragma once

namespace {

// The calling thread's current device is the context's for the duration of a call, whatever it was.
struct DeviceGuard {
  int before = -1;
  explicit DeviceGuard(int device) {
    int now = -1;
    if (cudaGetDevice(&now) == cudaSuccess && now != device && cudaSetDevice(device) == cudaSuccess) before = now;
  }
  ~DeviceGuard() {
    if (before >= 0) cudaSetDevice(before);
  }
};

size_t ca_smem_bytes(int n_seg) {
  return CA_STAGES * CA_STAGE_BYTES + CA_JOIN_BYTES + CA_JOBS * CA_Q_BYTES + sizeof(CaBook) + (size_t)n_seg * sizeof(CaSeg) + (size_t)(n_seg + 1) * sizeof(int);
}

size_t ct_smem_bytes(int n_seg) { return CT_BOOK_OFF + sizeof(CtBook) + (size_t)n_seg * sizeof(CaSeg) + (size_t)(n_seg + 1) * sizeof(int); }

// Elements that [rows, heads, dim] with the given strides spans.
long long span_of(long long rows, long long heads, long long dim, long long row, long long head) {
  return (rows - 1) * row + (heads - 1) * head + dim;
}
bool ranges_overlap(const void *a, long long na, const void *b, long long nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}
// No two elements of a tensor that is written share an address.
bool strides_disjoint(long long rows, long long heads, long long dim, long long row, long long head) {
  if (heads == 1) return rows == 1 || row >= dim;
  if (rows == 1) return head >= dim;
  return (head >= dim && row >= (heads - 1) * head + dim) || (row >= dim && head >= (rows - 1) * row + dim);
}
constexpr int MAX_ROWS = 1 << 30;              // rows that 32-bit counters walk in strides
constexpr long long MAX_STRIDE = 1LL << 39;    // elements of two bytes (a tensor map's strides are below 2^40 bytes)

constexpr long long CA_MAX_NUMBERS = 1LL << 30;    // key tiles are numbered in 32 bits

// The sizes and the type, which are all that the scratch depends on.  What passes keeps the layout's products within 64 bits.
asap_status check_cache_sizes(asap_ctx *ctx, const asap_cache_attention_args *p) {
  const char *who = "asap_cache_attention";
  if (!p) return fail(ctx, ASAP_ERR_INVALID, "%s: null arguments", who);
  if (p->B <= 0 || p->H <= 0 || p->kv_heads <= 0 || p->n_q <= 0 || p->max_q <= 0 || p->cache_rows <= 0)
    return fail(ctx, ASAP_ERR_INVALID, "%s: B, H, kv_heads, n_q, max_q and cache_rows must be positive", who);
  if (p->head_dim != 128) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: head_dim must be 128, got %d", who, p->head_dim);
  if (p->dtype != ASAP_BF16 && p->dtype != ASAP_FP16) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->H % p->kv_heads != 0) return fail(ctx, ASAP_ERR_INVALID, "%s: kv_heads must divide H", who);
  if (p->H > 65536) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: H above 65536", who);
  if (p->max_len < 0 || p->max_prefix < 0 || p->n_groups < 0 || p->max_len > p->cache_rows || p->max_prefix > p->cache_rows)
    return fail(ctx, ASAP_ERR_INVALID, "%s: need 0 <= max_len, max_prefix <= cache_rows and n_groups >= 0", who);
  if (p->max_q > p->n_q || p->n_groups > p->B) return fail(ctx, ASAP_ERR_INVALID, "%s: need max_q <= n_q and n_groups <= B", who);
  if ((long long)p->B + p->n_groups > CA_MAX_SEGMENTS)
    return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: at most %d sequences and groups in a call", who, CA_MAX_SEGMENTS);
  if ((long long)p->n_q * p->H > CA_MAX_NUMBERS / 2) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: n_q and H are too large together", who);
  return ASAP_OK;
}
asap_status check_cache_attention(asap_ctx *ctx, const asap_cache_attention_args *p) {
  const char *who = "asap_cache_attention";
  ASAP_TRY(check_cache_sizes(ctx, p));
  if (!(p->scale >= 0.f) || p->scale > 1e30f) return fail(ctx, ASAP_ERR_INVALID, "%s: scale must be finite and not negative", who);
  if (!p->q || !p->k || !p->v || !p->out || !p->start || !p->len) return fail(ctx, ASAP_ERR_INVALID, "%s: null q / k / v / out / start / len", who);
  if (p->n_groups > 0 && (!p->group_cu || !p->prefix_start || !p->prefix_len))
    return fail(ctx, ASAP_ERR_INVALID, "%s: n_groups needs group_cu, prefix_start and prefix_len", who);
  if (!p->q_cu && p->n_q != p->B) return fail(ctx, ASAP_ERR_INVALID, "%s: without q_cu there is one query row per sequence: n_q == B", who);
  if (!aligned16(p->q) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->out))
    return fail(ctx, ASAP_ERR_ALIGN, "%s: q / k / v / out must be 16-byte aligned", who);
  for (long long s : {(long long)p->q_row, (long long)p->q_head, (long long)p->out_row, (long long)p->out_head, (long long)p->kv_row, (long long)p->kv_head}) {
    if (s < 0 || s >= MAX_STRIDE) return fail(ctx, ASAP_ERR_INVALID, "%s: a stride is negative or too large", who);
    if (s % 8 != 0) return fail(ctx, ASAP_ERR_ALIGN, "%s: strides must be multiples of 8 elements", who);
  }
  if (!strides_disjoint(p->n_q, p->H, 128, p->out_row, p->out_head)) return fail(ctx, ASAP_ERR_INVALID, "%s: rows of out overlap", who);
  if ((p->cache_rows > 1 && p->kv_row < 128) || (p->kv_heads > 1 && p->kv_head < 128))
    return fail(ctx, ASAP_ERR_INVALID, "%s: the strides of k and v must be at least 128", who);
  const long long out_n = 2 * span_of(p->n_q, p->H, 128, p->out_row, p->out_head), q_n = 2 * span_of(p->n_q, p->H, 128, p->q_row, p->q_head),
                  kv_n = 2 * span_of(p->cache_rows, p->kv_heads, 128, p->kv_row, p->kv_head);
  if (ranges_overlap(p->out, out_n, p->q, q_n) || ranges_overlap(p->out, out_n, p->k, kv_n) || ranges_overlap(p->out, out_n, p->v, kv_n))
    return fail(ctx, ASAP_ERR_INVALID, "%s: out overlaps q, k or v", who);
  return ASAP_OK;
}

constexpr const char *CA_TOO_LARGE = "asap_cache_attention: max_q, max_len, max_prefix and the batch are too large together";

// Scratch of a call; `at` NULL: only its size.
struct CaLayout {
  size_t bytes = 0;
  int blocks[2] = {0, 0};        // of the streaming and of the tile kernel; 0: nothing to launch
  int pieces[2] = {0, 0};        // pieces of their work
  int rec_rows = 0;
  bool too_large = false;
  bool few = false;              // weights by ca_weight_few_kernel
  int own_lanes = 0, pre_lanes = 0;          // threads side by side on the keys
  long long own_blocks = 0, pre_blocks = 0;  // blocks of a sequence and of a prefix
};
CaLayout ca_layout(const asap_ctx *ctx, const asap_cache_attention_args *p, uint8_t *at, CacheArgs *a) {
  CaLayout l;
  const size_t entries = (size_t)p->n_q * p->H, n_seg = (size_t)p->B + p->n_groups;
  // no more blocks than there can be key tiles; no tile kernel where no segment can have more than 16 stacked rows
  const long long rep = p->H / p->kv_heads, heads = p->kv_heads, group_rows = p->n_groups > 0 && p->max_prefix > 0 ? p->n_q * rep : 0;
  // (heads that go together count less than the same heads one by one)
  auto numbers = [&](long long segs, long long rows, long long keys, auto work) {
    using WORK = decltype(work);
    return segs * ((rows + WORK::ROWS - 1) / WORK::ROWS) * ((keys + WORK::KEYS - 1) / WORK::KEYS + WORK::EXTRA) * heads;
  };
  auto at_most = [](long long n, long long most) { return (int)(n < 1 ? 1 : n < most ? n : most); };
  const long long own_rows = p->max_q * rep, S = StreamWork::ROWS;
  const long long streamed = numbers(p->B, 1, p->max_len, StreamWork{}) + (group_rows ? numbers(p->n_groups, 1, p->max_prefix, StreamWork{}) : 0);
  const long long tiled = (own_rows > S ? numbers(p->B, own_rows, p->max_len, TileWork{}) : 0) +
                          (group_rows > S ? numbers(1, group_rows + (long long)TileWork::ROWS * p->n_groups, p->max_prefix, TileWork{}) : 0);
  l.blocks[0] = at_most(streamed, 2LL * ctx->num_sms);
  if (tiled > 0) l.blocks[1] = at_most(tiled, ctx->num_sms);
  l.pieces[0] = at_most(streamed, 4LL * l.blocks[0]);
  l.pieces[1] = l.blocks[1];
  const long long group_max = group_rows > 0 ? (group_rows < S ? group_rows : S) : 0, own_max = own_rows < S ? own_rows : S;
  const long long rows_max = group_max > own_max ? group_max : own_max;
  l.rec_rows = (int)(4 * rows_max < S ? 4 * rows_max : S);           // (as many heads together as make up to 16 rows)
  l.too_large = streamed > CA_MAX_NUMBERS || tiled > CA_MAX_NUMBERS;
  if (p->weights) {
    const auto lanes_of = [](long long pairs) { return pairs <= 64 ? 64 : pairs <= 512 ? 16 : 4; };
    l.few = p->n_groups == 0 && (long long)p->max_q * p->H <= CA_FEW_PAIRS && p->max_len > 0;
    l.own_lanes = l.few ? CA_FEW_LANES : lanes_of((long long)p->max_q * p->H);
    l.pre_lanes = lanes_of((long long)p->n_q * p->H / (p->n_groups ? p->n_groups : 1));
    l.own_blocks = ((long long)p->max_len + 4 * l.own_lanes - 1) / (4 * l.own_lanes);
    l.pre_blocks = ((long long)p->max_prefix + 4 * l.pre_lanes - 1) / (4 * l.pre_lanes);
    l.too_large = l.too_large || l.own_blocks * p->B + l.pre_blocks * p->n_groups > CA_MAX_NUMBERS;
  }
  auto carve = [&](size_t bytes) {
    const size_t o = l.bytes;
    l.bytes = align_up(l.bytes + bytes, 256);
    return at + o;
  };
  const size_t rec[2] = {(size_t)2 * l.pieces[0] * l.rec_rows, (size_t)2 * l.pieces[1] * TileWork::ROWS};
  const long long own_off = p->n_groups ? ((long long)p->max_prefix + 127) / 128 * 128 : 0;
  const long long pitch = own_off + ((long long)p->max_len + 127) / 128 * 128;       // (a key tile is written whole)
  uint8_t *plan = carve((2 * (n_seg + 1) + 1) * 4), *rows = carve((size_t)p->n_q * sizeof(CaRow)), *rec_ml0 = carve(rec[0] * 8), *rec_ml1 = carve(rec[1] * 8),
          *full_ml = carve(2 * entries * 8), *rec_o0 = carve(rec[0] * 512), *rec_o1 = carve(rec[1] * 512), *full_o = carve(2 * entries * 512),
          *lse2 = carve(entries * 4), *logits = p->weights ? carve(entries * (size_t)pitch * 4) : nullptr;
  if (a) {
    a->plan = reinterpret_cast<int *>(plan); a->rows = reinterpret_cast<CaRow *>(rows);
    a->rec_ml[0] = reinterpret_cast<float2 *>(rec_ml0); a->rec_ml[1] = reinterpret_cast<float2 *>(rec_ml1);
    a->full_ml = reinterpret_cast<float2 *>(full_ml);
    a->rec_o[0] = reinterpret_cast<float *>(rec_o0); a->rec_o[1] = reinterpret_cast<float *>(rec_o1);
    a->full_o = reinterpret_cast<float *>(full_o); a->lse2 = reinterpret_cast<float *>(lse2);
    a->logits = reinterpret_cast<float *>(logits); a->pitch = pitch; a->own_off = (int)own_off;
    a->pieces[0] = l.pieces[0]; a->pieces[1] = l.pieces[1]; a->rec_rows = l.rec_rows;
  }
  return l;
}

// Keys or values [rows, heads, 128] with any strides, as four dimensions (64 columns, row, column half, head); box = 64 columns x box_rows rows x
// both halves x `heads`, 128-byte swizzle: in shared memory the halves of every head are blocks of box_rows x 128 bytes.
bool make_cache_map(asap_ctx *ctx, CUtensorMap *map, const void *ptr, const asap_cache_attention_args *p, uint32_t box_rows, uint32_t heads) {
  cuuint64_t dims[4] = {64, (cuuint64_t)p->cache_rows, 2, (cuuint64_t)p->kv_heads};
  cuuint64_t strides[3] = {(cuuint64_t)(p->cache_rows > 1 ? p->kv_row : 128) * 2, 128, (cuuint64_t)(p->kv_heads > 1 ? p->kv_head : 128) * 2};
  cuuint32_t box[4] = {64, box_rows, 2, heads};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return ctx->encode(map, p->dtype == ASAP_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(ptr),
                     dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Queries [n_q, H, 128] as five dimensions (64 columns, head of a key / value head, query row, column half, key / value head); box = a row
// tile of 128 stacked rows.  For H / kv_heads a divisor of 128.
bool make_query_map(asap_ctx *ctx, CUtensorMap *map, const asap_cache_attention_args *p) {
  const cuuint64_t rep = p->H / p->kv_heads;
  cuuint64_t dims[5] = {64, rep, (cuuint64_t)p->n_q, 2, (cuuint64_t)p->kv_heads};
  const cuuint64_t row = p->n_q > 1 ? p->q_row : 128, head = p->H > 1 ? p->q_head : 128;
  cuuint64_t strides[4] = {head * 2, row * 2, 128, rep * head * 2};
  cuuint32_t box[5] = {64, (cuuint32_t)rep, 128 / (cuuint32_t)rep, 2, 1};
  cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return ctx->encode(map, p->dtype == ASAP_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(p->q),
                     dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" {

asap_status asap_rope_make(asap_rope_plan *plan, int32_t rot_dim, int32_t interleaved, int32_t scaling, double theta, double factor,
                           double original_positions, double fast, double slow) {
  const char *who = "asap_rope_make";
  if (!plan) return fail(nullptr, ASAP_ERR_INVALID, "%s: null plan", who);
  if (rot_dim <= 0 || rot_dim % 2 != 0 || rot_dim > 2 * ROPE_MAX_PAIRS)
    return fail(nullptr, ASAP_ERR_UNSUPPORTED, "%s: rot_dim must be even, 2 .. %d", who, 2 * ROPE_MAX_PAIRS);
  if (scaling < ASAP_ROPE_PLAIN || scaling > ASAP_ROPE_BANDS) return fail(nullptr, ASAP_ERR_INVALID, "%s: unknown scaling %d", who, scaling);
  if (!(theta > 1.0) || !(theta < 1e300)) return fail(nullptr, ASAP_ERR_INVALID, "%s: theta must be above 1", who);
  if (scaling != ASAP_ROPE_PLAIN && (!(factor >= 1.0) || !(factor < 1e9))) return fail(nullptr, ASAP_ERR_INVALID, "%s: factor must be at least 1", who);
  if (scaling == ASAP_ROPE_NTK && rot_dim <= 2) return fail(nullptr, ASAP_ERR_UNSUPPORTED, "%s: NTK scaling needs rot_dim > 2", who);
  if (scaling == ASAP_ROPE_YARN || scaling == ASAP_ROPE_BANDS)
    if (!(original_positions > 0.0) || !(original_positions < 1e15) || !(slow > 0.0) || !(fast > slow) || !(fast < 1e15))
      return fail(nullptr, ASAP_ERR_INVALID, "%s: need original_positions > 0 and 0 < slow < fast", who);
  const double two_pi = 6.283185307179586476925286766559;
  const int n = rot_dim / 2;
  memset(plan, 0, sizeof(*plan));
  plan->n_pairs = n; plan->interleaved = interleaved ? 1 : 0; plan->magnitude = 1.f;
  if (scaling == ASAP_ROPE_NTK) theta *= pow(factor, (double)rot_dim / (rot_dim - 2));
  double low = 0.0, high = 0.0;
  if (scaling == ASAP_ROPE_YARN) {
    // the pair that turns r times over the original positions: original / (2 pi theta^(i / n)) = r
    auto at = [&](double r) { return n * log(original_positions / (r * two_pi)) / log(theta); };
    low = fmax(floor(at(fast)), 0.0);
    high = fmin(ceil(at(slow)), (double)(rot_dim - 1));
    plan->magnitude = (float)(0.1 * log(factor) + 1.0);
  }
  for (int i = 0; i < n; ++i) {
    double t = pow(theta, -(double)i / n) / two_pi;
    if (scaling == ASAP_ROPE_LINEAR) t /= factor;
    if (scaling == ASAP_ROPE_YARN || scaling == ASAP_ROPE_BANDS) {
      // share of the pair that is divided
      double x = scaling == ASAP_ROPE_YARN ? (i - low) / fmax(high - low, 0.001) : 1.0 - (original_positions * t - slow) / (fast - slow);
      x = fmin(fmax(x, 0.0), 1.0);
      t = t * (1.0 - x) + t / factor * x;
    }
    plan->turns[i] = (uint64_t)(t * 18446744073709551616.0);     // (t < 1 / (2 pi): no overflow)
  }
  return ASAP_OK;
}

asap_status asap_rope(asap_ctx *ctx, const asap_rope_plan *plan, const asap_rope_args *p, void *stream) {
  const char *who = "asap_rope";
  if (!ctx) return fail(nullptr, ASAP_ERR_INVALID, "null context");
  ctx->err[0] = 0;
  if (!plan || !p) return fail(ctx, ASAP_ERR_INVALID, "%s: null plan / arguments", who);
  if (plan->n_pairs <= 0 || plan->n_pairs > ROPE_MAX_PAIRS) return fail(ctx, ASAP_ERR_INVALID, "%s: the plan was not made by asap_rope_make", who);
  if (p->n_rows < 0) return fail(ctx, ASAP_ERR_INVALID, "%s: n_rows is negative", who);
  if (p->head_dim <= 0 || p->head_dim % 8 != 0 || p->head_dim > 256)
    return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of 8 up to 256, got %d", who, p->head_dim);
  if (2 * plan->n_pairs > p->head_dim) return fail(ctx, ASAP_ERR_INVALID, "%s: the plan rotates %d elements of a head of %d", who, 2 * plan->n_pairs, p->head_dim);
  if (p->dtype != ASAP_BF16 && p->dtype != ASAP_FP16) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, p->dtype);
  if (p->n_tensors <= 0 || p->n_tensors > 4 || !p->tensors) return fail(ctx, ASAP_ERR_INVALID, "%s: 1 .. 4 tensors", who);
  if (p->n_rows > 0 && !p->pos) return fail(ctx, ASAP_ERR_INVALID, "%s: null pos", who);
  RopeArgs a;
  for (int i = 0; i < p->n_tensors; ++i) {
    const asap_rope_tensor &t = p->tensors[i];
    if (t.heads <= 0) return fail(ctx, ASAP_ERR_INVALID, "%s: heads of tensor %d must be positive", who, i);
    if (t.heads > 65536) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: heads of tensor %d above 65536", who, i);
    if (p->n_rows > 0 && (!t.src || !t.dst)) return fail(ctx, ASAP_ERR_INVALID, "%s: null tensor %d", who, i);
    if (t.mapped && p->n_rows > 0 && (!p->dst_map || p->dst_rows <= 0)) return fail(ctx, ASAP_ERR_INVALID, "%s: tensor %d is mapped: dst_map and dst_rows are needed", who, i);
    if (!aligned16(t.src) || !aligned16(t.dst)) return fail(ctx, ASAP_ERR_ALIGN, "%s: tensor %d is not 16-byte aligned", who, i);
    for (long long s : {(long long)t.src_row, (long long)t.src_head, (long long)t.dst_row, (long long)t.dst_head}) {
      if (s < 0 || s >= MAX_STRIDE) return fail(ctx, ASAP_ERR_INVALID, "%s: a stride of tensor %d is negative or too large", who, i);
      if (s % 8 != 0) return fail(ctx, ASAP_ERR_ALIGN, "%s: strides must be multiples of 8 elements (tensor %d)", who, i);
    }
    if (p->n_rows > 0) {
      const long long dst_rows = t.mapped ? p->dst_rows : p->n_rows;
      if (!strides_disjoint(dst_rows, t.heads, p->head_dim, t.dst_row, t.dst_head))
        return fail(ctx, ASAP_ERR_INVALID, "%s: rows of destination %d overlap", who, i);
      const bool same = t.src == t.dst && t.src_row == t.dst_row && t.src_head == t.dst_head && !t.mapped;
      if (!same && ranges_overlap(t.src, 2 * span_of(p->n_rows, t.heads, p->head_dim, t.src_row, t.src_head), t.dst,
                                  2 * span_of(dst_rows, t.heads, p->head_dim, t.dst_row, t.dst_head)))
        return fail(ctx, ASAP_ERR_INVALID, "%s: source and destination %d overlap without being the same", who, i);
    }
    // (others may interleave with this one, as the parts of a packed projection do; the same start is no layout)
    for (int j = 0; j < i && p->n_rows > 0; ++j) {
      const asap_rope_tensor &u = p->tensors[j];
      if (u.dst == t.dst || u.src == t.dst || u.dst == t.src) return fail(ctx, ASAP_ERR_INVALID, "%s: destination of tensor %d or %d is a tensor of the other", who, j, i);
    }
    RopeTensor &r = a.t[i];
    r.src = static_cast<const uint16_t *>(t.src); r.dst = static_cast<uint16_t *>(t.dst);
    r.heads = t.heads; r.rotate = t.rotate ? 1 : 0; r.mapped = t.mapped ? 1 : 0;
    r.src_row = t.src_row; r.src_head = t.src_head; r.dst_row = t.dst_row; r.dst_head = t.dst_head;
  }
  if (p->n_rows == 0) return ASAP_OK;
  a.n_tensors = p->n_tensors; a.n_rows = p->n_rows; a.head_dim = p->head_dim; a.n_pairs = plan->n_pairs; a.interleaved = plan->interleaved ? 1 : 0;
  a.dst_rows = p->dst_rows; a.magnitude = plan->magnitude; a.sign = p->inverse ? -1.f : 1.f; a.pos = p->pos; a.map = p->dst_map;
  memcpy(a.turns, plan->turns, sizeof(a.turns));
  long long blocks = 0;
  for (int i = 0; i < p->n_tensors; ++i) {
    RopeTensor &t = a.t[i];
    t.rows = 1;
    if (p->n_rows >= 16 * ctx->num_sms) t.rows = t.heads >= 128 ? 1 : t.heads > 128 / ROPE_MAX_ROWS ? 128 / t.heads : ROPE_MAX_ROWS;
    t.first_block = (int)blocks;
    blocks += ((long long)p->n_rows + t.rows - 1) / t.rows;
  }
  if (blocks > 0x7fffffffLL) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: too many rows", who);
  const bool vec = plan->n_pairs % (plan->interleaved ? 4 : 8) == 0;
  DeviceGuard guard(ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool f16 = p->dtype == ASAP_FP16;
  mark(ctx, "rope", st);
  launch_pdl(f16 ? (vec ? rope_kernel<true, true> : rope_kernel<true, false>) : (vec ? rope_kernel<false, true> : rope_kernel<false, false>),
             dim3((unsigned)blocks), dim3(ROPE_THREADS), 0, st, a);
  return finish(ctx, after_launch(ctx, "rope"), st);
}

size_t asap_cache_attention_scratch_bytes(const asap_ctx *ctx, const asap_cache_attention_args *p) {
  if (!ctx || check_cache_sizes(nullptr, p) != ASAP_OK) return 0;
  const CaLayout layout = ca_layout(ctx, p, nullptr, nullptr);
  if (!layout.too_large) return layout.bytes;
  fail(nullptr, ASAP_ERR_UNSUPPORTED, CA_TOO_LARGE);
  return 0;
}

asap_status asap_cache_attention(asap_ctx *ctx, const asap_cache_attention_args *p, void *scratch, size_t scratch_bytes, void *stream) {
  if (!ctx) return fail(nullptr, ASAP_ERR_INVALID, "null context");
  ctx->err[0] = 0;
  ASAP_TRY(check_cache_attention(ctx, p));
  CacheArgs a;
  const CaLayout layout = ca_layout(ctx, p, static_cast<uint8_t *>(scratch), &a);
  if (layout.too_large) return fail(ctx, ASAP_ERR_UNSUPPORTED, CA_TOO_LARGE);
  if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255u) != 0 || scratch_bytes < layout.bytes)
    return fail(ctx, ASAP_ERR_WORKSPACE, "asap_cache_attention: scratch is null, not 256-byte aligned or smaller than asap_cache_attention_scratch_bytes");
  CaMaps maps;
  CUtensorMap tile_k = {}, tile_v = {}, tile_q = {};
  bool made = true;
  for (int b = 0; b < 3; ++b) {                  // (boxes of more heads than there are stand unused)
    const uint32_t heads = p->kv_heads >= 1 << b ? 1u << b : 1u;
    made = made && make_cache_map(ctx, &maps.k[b], p->k, p, StreamWork::KEYS / heads, heads) && make_cache_map(ctx, &maps.v[b], p->v, p, StreamWork::KEYS / heads, heads);
  }
  if (layout.blocks[1]) made = made && make_cache_map(ctx, &tile_k, p->k, p, TileWork::KEYS, 1) && make_cache_map(ctx, &tile_v, p->v, p, TileWork::KEYS, 1);
  // (rows or heads that share an address, as a broadcast view has them, are gathered)
  const int rep = p->H / p->kv_heads;
  a.q_tiled = layout.blocks[1] && 128 % rep == 0 && (p->n_q == 1 || p->q_row >= 128) && (p->H == 1 || p->q_head >= 128);
  tile_q = tile_k;
  if (a.q_tiled) made = made && make_query_map(ctx, &tile_q, p);
  if (!made) return fail(ctx, ASAP_ERR_CUDA, "cuTensorMapEncodeTiled failed for k / v");
  a.B = p->B; a.G = p->n_groups; a.H = p->H; a.kv = p->kv_heads; a.rep = p->H / p->kv_heads;
  a.n_q = p->n_q; a.max_q = p->max_q; a.max_len = p->max_len; a.max_prefix = p->max_prefix; a.cache_rows = p->cache_rows;
  a.q_row = p->q_row; a.q_head = p->q_head; a.out_row = p->out_row; a.out_head = p->out_head;
  a.q_cu = p->q_cu; a.start = p->start; a.len = p->len; a.group_cu = p->group_cu; a.prefix_start = p->prefix_start; a.prefix_len = p->prefix_len;
  a.q = static_cast<const uint16_t *>(p->q); a.v = static_cast<const uint16_t *>(p->v); a.kv_row = p->kv_row; a.kv_head = p->kv_head;
  a.out = static_cast<uint16_t *>(p->out); a.lse = p->lse; a.weights = p->weights;
  a.scale_log2 = 1.4426950408889634f * (p->scale > 0.f ? p->scale : 1.0f / sqrtf(128.f));
  a.status = ctx->status; a.wait_limit = ctx->wait_limit; a.work = ctx->cnt_work + 4;
  const bool f16 = p->dtype == ASAP_FP16;
  DeviceGuard guard(ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (layout.blocks[1]) {
    mark(ctx, "cache_tile", st);
    launch_pdl(f16 ? (p->weights ? ca_tile_kernel<true, true> : ca_tile_kernel<true, false>) : (p->weights ? ca_tile_kernel<false, true> : ca_tile_kernel<false, false>), dim3(layout.blocks[1]), dim3(CT_THREADS), ct_smem_bytes(p->B + p->n_groups), st,
               tile_k, tile_v, tile_q, a);
    ASAP_TRY(after_launch(ctx, "cache_tile"));
  }
  mark(ctx, "cache_stream", st);
  launch_pdl(f16 ? ca_stream_kernel<true> : ca_stream_kernel<false>, dim3(layout.blocks[0]), dim3(CA_THREADS), ca_smem_bytes(p->B + p->n_groups), st,
             maps, a);
  ASAP_TRY(after_launch(ctx, "cache_stream"));
  a.join_behind = layout.few ? 1 : 0;
  if (layout.few) {
    mark(ctx, "cache_weight", st);
    launch_pdl(ca_weight_few_kernel, dim3((unsigned)(layout.own_blocks * p->B)), dim3(CA_WEIGHT_THREADS), 0, st, a, (int)layout.own_blocks);
    ASAP_TRY(after_launch(ctx, "cache_weight"));
  }
  mark(ctx, "cache_join", st);
  // (the form with the most blocks that the device holds at a time.  Two heads: 1 x 32 heads 14 -> 8 us, 5 rows of up to 150 partial results 17 ->
  // 8, but 128 rows 21 -> 62; eight: 61 rows 16 -> 12; sixteen: 128 rows 18.5 -> 16.5)
  const auto blocks_of = [&](int heads) { return (long long)p->n_q * ((p->H + heads - 1) / heads); };
  int heads = CA_JOIN_HEADS;
  for (int few_heads : {16, 8, 2})
    if (blocks_of(few_heads) <= 2LL * ctx->num_sms) heads = few_heads;
  const int rows = heads == CA_JOIN_HEADS && p->n_q >= 4 * ctx->num_sms ? 4 : 1;
  void (*join)(CacheArgs) = heads == 2    ? (f16 ? ca_join_kernel<true, 2, 1> : ca_join_kernel<false, 2, 1>)
                          : heads == 8    ? (f16 ? ca_join_kernel<true, 8, 1> : ca_join_kernel<false, 8, 1>)
                          : heads == 16   ? (f16 ? ca_join_kernel<true, 16, 1> : ca_join_kernel<false, 16, 1>)
                          : rows == 1     ? (f16 ? ca_join_kernel<true, 32, 1> : ca_join_kernel<false, 32, 1>)
                                          : (f16 ? ca_join_kernel<true, 32, 4> : ca_join_kernel<false, 32, 4>);
  launch_pdl(join, dim3((p->n_q + rows - 1) / rows, (p->H + heads - 1) / heads), dim3(rows > 1 ? CA_JOIN_MANY_THREADS : CA_JOIN_THREADS), 0, st, a);
  ASAP_TRY(after_launch(ctx, "cache_join"));
  const long long weight_blocks = layout.pre_blocks * p->n_groups + layout.own_blocks * p->B;
  if (p->weights && !layout.few && weight_blocks > 0) {
    mark(ctx, "cache_weight", st);
    launch_pdl(ca_weight_kernel, dim3((unsigned)weight_blocks), dim3(CA_WEIGHT_THREADS), 0, st, a, (int)layout.pre_blocks, layout.pre_lanes,
               (int)layout.own_blocks, layout.own_lanes);
    ASAP_TRY(after_launch(ctx, "cache_weight"));
  }
  return finish(ctx, ASAP_OK, st);
}

asap_status asap_cache_evict(asap_ctx *ctx, const asap_cache_evict_args *p, void *stream) {
  const char *who = "asap_cache_evict";
  if (!ctx) return fail(nullptr, ASAP_ERR_INVALID, "null context");
  ctx->err[0] = 0;
  if (!p) return fail(ctx, ASAP_ERR_INVALID, "%s: null arguments", who);
  if (p->B <= 0 || p->max_len <= 0 || p->keep <= 0 || p->rows <= 0 || p->dst_rows <= 0)
    return fail(ctx, ASAP_ERR_INVALID, "%s: B, max_len, keep, rows and dst_rows must be positive", who);
  if (p->keep > MAX_ROWS || p->max_len > MAX_ROWS) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: keep and max_len at most 2^30", who);
  if (p->sink < 0 || p->recent < 0 || (long long)p->sink + p->recent > p->keep)
    return fail(ctx, ASAP_ERR_INVALID, "%s: need 0 <= sink, recent and sink + recent <= keep", who);
  if (p->B > 65535) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: at most 65535 sequences", who);
  if (!p->start || !p->len || !p->weights || !p->keep_idx || !p->new_len)
    return fail(ctx, ASAP_ERR_INVALID, "%s: null start / len / weights / keep_idx / new_len", who);
  if (p->n_tensors < 0 || p->n_tensors > EV_MAX_TENSORS) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: 0 .. %d tensors per call", who, EV_MAX_TENSORS);
  if (p->n_tensors > 0 && (!p->src || !p->dst)) return fail(ctx, ASAP_ERR_INVALID, "%s: null src / dst", who);
  if (p->n_tensors > 0 && (p->row_bytes == 0 || p->row_bytes % 16 != 0 || p->row_bytes / 16 > 0x7fffff))
    return fail(ctx, ASAP_ERR_ALIGN, "%s: row_bytes must be a positive multiple of 16", who);
  const long long src_n = (long long)p->rows * (long long)p->row_bytes, dst_n = (long long)p->dst_rows * (long long)p->row_bytes;
  EvictMoveArgs mv;
  bool in_place = false;
  for (int t = 0; t < p->n_tensors; ++t) {
    if (!p->src[t] || !p->dst[t]) return fail(ctx, ASAP_ERR_INVALID, "%s: null tensor %d", who, t);
    if (!aligned16(p->src[t]) || !aligned16(p->dst[t])) return fail(ctx, ASAP_ERR_ALIGN, "%s: tensor %d is not 16-byte aligned", who, t);
    const bool same = p->src[t] == p->dst[t];
    if (t > 0 && same != in_place) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: either all tensors move in place or none", who);
    in_place = same;
    mv.src[t] = static_cast<const uint4 *>(p->src[t]);
    mv.dst[t] = static_cast<uint4 *>(p->dst[t]);
  }
  for (int t = 0; t < p->n_tensors && !in_place; ++t)
    for (int u = 0; u < p->n_tensors; ++u)
      if (ranges_overlap(p->src[u], src_n, p->dst[t], dst_n)) return fail(ctx, ASAP_ERR_INVALID, "%s: destination %d overlaps source %d", who, t, u);
  for (int t = 0; t < p->n_tensors; ++t)
    for (int u = t + 1; u < p->n_tensors; ++u)
      if (ranges_overlap(p->dst[t], dst_n, p->dst[u], dst_n)) return fail(ctx, ASAP_ERR_INVALID, "%s: destinations %d and %d overlap", who, t, u);
  const bool meta_in_place = (p->dst_weights && p->dst_weights == p->weights) || (p->dst_pos && p->dst_pos == p->pos);
  if ((in_place || meta_in_place) && p->dst_start) return fail(ctx, ASAP_ERR_INVALID, "%s: in place the rows stay behind start: dst_start must be NULL", who);
  if ((in_place || meta_in_place) && p->rows != p->dst_rows) return fail(ctx, ASAP_ERR_INVALID, "%s: in place rows == dst_rows", who);
  if ((p->dst_weights && p->dst_weights != p->weights && ranges_overlap(p->weights, 4LL * p->rows, p->dst_weights, 4LL * p->dst_rows)) ||
      (p->dst_pos && p->pos && p->dst_pos != p->pos && ranges_overlap(p->pos, 4LL * p->rows, p->dst_pos, 4LL * p->dst_rows)))
    return fail(ctx, ASAP_ERR_INVALID, "%s: dst_weights / dst_pos overlap weights / pos without being the same", who);
  EvictArgs a;
  a.B = p->B; a.max_len = p->max_len; a.keep = p->keep; a.sink = p->sink; a.recent = p->recent; a.rows = p->rows; a.dst_rows = p->dst_rows;
  a.start = p->start; a.len = p->len; a.dst_start = p->dst_start; a.weights = p->weights; a.pos = p->pos; a.keep_idx = p->keep_idx;
  a.new_len = p->new_len; a.status = ctx->status;
  // (where max_len <= keep every sequence stays whole, and its rows are not ranked)
  const long long rounds = ((long long)p->B * EV_CLUSTER + ctx->num_sms - 1) / ctx->num_sms;
  const bool cluster = ctx->evict_cluster && p->max_len > p->keep && p->max_len >= (rounds == 1 ? EV_CLUSTER_MIN : rounds * EV_CLUSTER_MIN_ROUND);
  const long long share = p->max_len > p->keep ? (((long long)p->max_len + (cluster ? EV_CLUSTER : 1) - 1) / (cluster ? EV_CLUSTER : 1) + 31) / 32 * 32 : 0;
  a.cached = share * 4 <= EV_KEYS_BYTES ? (int)share : 0;
  DeviceGuard guard(ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  mark(ctx, cluster ? "evict_select_cluster" : "evict_select", st);
  if (cluster)
    launch_pdl_cluster_z(evict_select_kernel<true>, dim3(1, p->B, EV_CLUSTER), dim3(EV_THREADS), (size_t)a.cached * 4, st, EV_CLUSTER, a);
  else
    launch_pdl(evict_select_kernel<false>, dim3(1, p->B), dim3(EV_THREADS), (size_t)a.cached * 4, st, a);
  ASAP_TRY(after_launch(ctx, "evict_select"));
  const bool meta = p->dst_weights || p->dst_pos;
  if (p->n_tensors > 0 || meta) {
    mv.keep_idx = p->keep_idx; mv.start = p->start; mv.dst_start = p->dst_start; mv.keep = p->keep; mv.n_tensors = p->n_tensors;
    mv.row_vecs = p->n_tensors > 0 ? (int)(p->row_bytes / 16) : 1;
    mv.weights = p->weights; mv.pos = p->pos; mv.dst_weights = p->dst_weights; mv.dst_pos = p->dst_pos;
    const unsigned layers = p->n_tensors + (meta ? 1 : 0);
    mark(ctx, "evict_move", st);
    mv.in_order = meta_in_place ? 1 : 0;
    if (in_place)
      launch_pdl(evict_in_place_kernel, dim3((mv.row_vecs + 15) / 16, p->B, layers), dim3(EV_MOVE_THREADS), 0, st, mv);
    else {
      mv.warp_rows = mv.row_vecs < 256 ? 256 / mv.row_vecs : 1;
      const int block_rows = mv.warp_rows * (EV_MOVE_THREADS / 32);
      const int move_blocks = (p->keep + block_rows - 1) / block_rows, meta_blocks = meta ? (p->keep + EV_MOVE_THREADS - 1) / EV_MOVE_THREADS : 0;
      launch_pdl(evict_move_kernel, dim3(p->n_tensors == 0 || meta_blocks > move_blocks ? meta_blocks : move_blocks, p->B, layers), dim3(EV_MOVE_THREADS), 0, st, mv);
    }
    ASAP_TRY(after_launch(ctx, "evict_move"));
  }
  return finish(ctx, ASAP_OK, st);
}

asap_status asap_cache_slot(asap_ctx *ctx, const asap_cache_slot_args *p, void *stream) {
  const char *who = "asap_cache_slot";
  if (!ctx) return fail(nullptr, ASAP_ERR_INVALID, "null context");
  ctx->err[0] = 0;
  if (!p) return fail(ctx, ASAP_ERR_INVALID, "%s: null arguments", who);
  if (p->B <= 0 || p->capacity <= 0 || p->rows <= 0) return fail(ctx, ASAP_ERR_INVALID, "%s: B, capacity and rows must be positive", who);
  if (p->capacity > MAX_ROWS) return fail(ctx, ASAP_ERR_UNSUPPORTED, "%s: capacity at most 2^30", who);
  if (p->sink < 0 || p->recent < 0 || (long long)p->sink + p->recent >= p->capacity)
    return fail(ctx, ASAP_ERR_INVALID, "%s: need 0 <= sink, recent and sink + recent < capacity", who);
  if (!p->start || !p->len || !p->weights || !p->pos || !p->new_pos || !p->row)
    return fail(ctx, ASAP_ERR_INVALID, "%s: null start / len / weights / pos / new_pos / row", who);
  SlotArgs a;
  a.B = p->B; a.capacity = p->capacity; a.sink = p->sink; a.recent = p->recent; a.rows = p->rows; a.start = p->start; a.len = p->len;
  a.weights = p->weights; a.pos = p->pos; a.new_pos = p->new_pos; a.row = p->row; a.status = ctx->status;
  DeviceGuard guard(ctx->device);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  mark(ctx, "slot", st);
  launch_pdl(slot_kernel, dim3(p->B), dim3(SLOT_THREADS), 0, st, a);
  return finish(ctx, after_launch(ctx, "slot"), st);
}

}  // extern "C"
