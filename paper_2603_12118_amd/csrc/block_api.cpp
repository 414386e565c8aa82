// C entry points of the LLM task's layer behind its attention (argument checks; the kernels are in block.hip and packed.hip).
#include <string>

#include "block.h"

using namespace cs;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
cs_status invalid(const char* who, const char* what) { return fail(CS_ERR_INVALID_ARG, std::string(who) + ": " + what); }
cs_status unsupported(const char* who, const char* what) { return fail(CS_ERR_UNSUPPORTED, std::string(who) + ": " + what); }
bool is_dtype(int32_t d) { return d == CS_F32 || d == CS_BF16; }
bool is_flag(int32_t v) { return v == 0 || v == 1; }

constexpr int64_t MAX_ROWS = (int64_t)1 << 31;

// rows of `width` values of `size` bytes, `row` values apart
cs_status check_rows(const char* who, const char* name, const void* p, int64_t row, int64_t width, int size) {
  if (!p || !aligned(p, 16)) return invalid(who, (std::string("NULL or misaligned ") + name).c_str());
  if (row < width || row > (int64_t)1 << 40) return invalid(who, (std::string("rows overlap or lie too far apart: ") + name).c_str());
  if (row * size % 16) return unsupported(who, (std::string("rows must be multiples of 16 bytes apart: ") + name).c_str());
  return CS_OK;
}

cs_status check_n_rows(const char* who, int64_t n_rows) {
  if (n_rows < 0) return invalid(who, "negative size");
  return n_rows >= MAX_ROWS ? unsupported(who, "at most 2^31 - 1 rows") : CS_OK;
}

cs_status check_workspace(const char* who, const void* workspace, size_t bytes, size_t need) {
  if (need && (!workspace || !aligned(workspace, 16))) return invalid(who, "NULL or misaligned workspace");
  if (bytes < need)
    return fail(CS_ERR_WORKSPACE, std::string(who) + ": needs " + std::to_string(need) + " bytes of workspace, got " + std::to_string(bytes));
  return CS_OK;
}

cs_status norm_residual(const cs_norm_config* c, const void* x, int64_t x_row, const void* residual, int64_t residual_row, const void* gate,
                        int64_t gate_row, const float* post_gain, const float* post_bias, const float* pre_gain, const float* pre_bias, void* r,
                        int64_t r_row, void* y, int64_t y_row, int64_t n_rows, void* stream) {
  const char* who = "cs_norm_residual";
  if (!c) return invalid(who, "NULL configuration");
  if (c->struct_size != sizeof(cs_norm_config)) return invalid(who, "config.struct_size mismatch");
  if (c->norm != CS_NORM_RMS && c->norm != CS_NORM_LAYER) return invalid(who, "norm");
  if (!is_dtype(c->dtype) || !is_dtype(c->residual_dtype)) return invalid(who, "dtype");
  if (c->gate < 0 || c->gate > 2) return invalid(who, "gate must be 0, 1 or 2");
  if (!(c->eps >= 0)) return invalid(who, "eps");
  if (!(c->residual_scale - c->residual_scale == 0) || !(c->block_scale - c->block_scale == 0)) return invalid(who, "scales must be finite");
  if (c->width <= 0) return invalid(who, "width");
  if (c->width % 8 || c->width > 16384) return unsupported(who, "width must be a multiple of 8, at most 16384");
  if (cs_status st = check_n_rows(who, n_rows)) return st;
  if (n_rows == 0) return CS_OK;
  const int size = c->dtype == CS_BF16 ? 2 : 4, rsize = c->residual_dtype == CS_BF16 ? 2 : 4;
  if (cs_status st = check_rows(who, "x", x, x_row, c->width, size)) return st;
  if (cs_status st = check_rows(who, "residual", residual, residual_row, c->width, rsize)) return st;
  if (cs_status st = check_rows(who, "r", r, r_row, c->width, rsize)) return st;
  if (cs_status st = check_rows(who, "y", y, y_row, c->width, size)) return st;
  if (c->gate)
    if (cs_status st = check_rows(who, "gate", gate, c->gate == 2 ? gate_row : c->width, c->width, size)) return st;
  if (!pre_gain) return invalid(who, "NULL pre_gain");
  if (post_bias && !post_gain) return invalid(who, "post_bias without post_gain");
  if (!aligned(post_gain, 16) || !aligned(post_bias, 16) || !aligned(pre_gain, 16) || !aligned(pre_bias, 16)) return invalid(who, "misaligned gains or biases");
  NormResidualArgs a = {};
  a.x = x; a.residual = residual; a.gate = c->gate ? gate : nullptr; a.r_out = r; a.y = y;
  a.x_row = x_row; a.residual_row = residual_row; a.gate_row = c->gate == 2 ? gate_row : 0; a.r_row = r_row; a.y_row = y_row;
  a.post_gain = post_gain; a.post_bias = post_bias; a.pre_gain = pre_gain; a.pre_bias = pre_bias;
  a.n_rows = n_rows; a.width = c->width;
  a.eps = c->eps; a.residual_scale = c->residual_scale; a.block_scale = c->block_scale;
  return launch_norm_residual(a, c->norm == CS_NORM_LAYER, c->dtype, c->residual_dtype, static_cast<hipStream_t>(stream));
}

cs_status check_weights(const char* who, const cs_weights_config* c, PackedShape& shape) {
  if (!c) return invalid(who, "NULL configuration");
  if (c->struct_size != sizeof(cs_weights_config)) return invalid(who, "config.struct_size mismatch");
  if (c->format != CS_WEIGHTS_E2M1 && c->format != CS_WEIGHTS_BF16) return invalid(who, "format");
  if (c->matrices <= 0 || c->n <= 0 || c->k <= 0) return invalid(who, "sizes");
  if (c->k % 32) return unsupported(who, "k must be a multiple of 32");
  if (c->n > 1 << 24 || c->k > 1 << 24 || c->matrices > 1 << 20) return unsupported(who, "n and k at most 2^24, at most 2^20 matrices");
  shape = packed_shape(c->format, c->matrices, c->n, c->k);
  if ((double)c->matrices * (double)matrix_bytes(shape) > 1e15) return unsupported(who, "more bytes than there are");
  return CS_OK;
}

cs_status weights(const char* who, const cs_weights_config* c, const void* w, int64_t w_row, int64_t w_matrix, int32_t dtype, const void* packed,
                  int32_t* err, PackArgs& a) {
  if (cs_status st = check_weights(who, c, a.shape)) return st;
  if (!is_dtype(dtype)) return invalid(who, "dtype");
  const int size = dtype == CS_BF16 ? 2 : 4;
  if (cs_status st = check_rows(who, "w", w, w_row, c->k, size)) return st;
  if (w_matrix < 0 || w_matrix > (int64_t)1 << 50) return invalid(who, "matrices lie too far apart");
  if (c->matrices > 1 && w_matrix * size % 16) return unsupported(who, "matrices must be multiples of 16 bytes apart");
  if (!packed || !aligned(packed, 16)) return invalid(who, "NULL or misaligned packed weights");
  if (!aligned(err, 4)) return invalid(who, "misaligned flag");
  a.w = w; a.w_row = w_row; a.w_matrix = w_matrix;
  a.packed = static_cast<unsigned char*>(const_cast<void*>(packed));
  a.err = err;
  return CS_OK;
}

cs_status linear_args(const char* who, const cs_weights_config* c, int64_t n_rows, LinearArgs& a, size_t& need) {
  if (cs_status st = check_weights(who, c, a.shape)) return st;
  if (c->matrices != 1) return invalid(who, "one matrix expected");
  if (cs_status st = check_n_rows(who, n_rows)) return st;
  a.n_rows = n_rows;
  need = 0;
  return n_rows ? plan_linear_packed(a, need) : CS_OK;
}

cs_status linear_packed(const cs_weights_config* c, const void* packed, const void* x, int64_t x_row, const float* bias, void* out,
                        int64_t out_row, int32_t out_dtype, int64_t n_rows, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "cs_linear_packed";
  LinearArgs a = {};
  size_t need = 0;
  if (cs_status st = linear_args(who, c, n_rows, a, need)) return st;
  if (!is_dtype(out_dtype)) return invalid(who, "out_dtype");
  if (n_rows == 0) return CS_OK;
  if (!packed || !aligned(packed, 16)) return invalid(who, "NULL or misaligned packed weights");
  if (cs_status st = check_rows(who, "x", x, x_row, c->k, 2)) return st;
  if (n_rows > 1 && x_row > 1 << 22) return unsupported(who, "rows of x at most 2^22 elements apart");
  if (!out || !aligned(out, out_dtype == CS_BF16 ? 2 : 4)) return invalid(who, "NULL or misaligned out");
  if (out_row < c->n || out_row > (int64_t)1 << 40) return invalid(who, "rows overlap or lie too far apart: out");
  if (!aligned(bias, 4)) return invalid(who, "misaligned bias");
  if (cs_status st = check_workspace(who, workspace, workspace_bytes, need)) return st;
  a.packed = static_cast<const unsigned char*>(packed);
  a.x = static_cast<const bf16_t*>(x); a.x_row = x_row; a.bias = bias; a.out = out; a.out_row = out_row;
  return launch_linear_packed(a, out_dtype, workspace, static_cast<hipStream_t>(stream));
}

cs_status moe_args(const char* who, const cs_moe_config* c, int64_t n_rows, MoeArgs& a) {
  if (!c) return invalid(who, "NULL configuration");
  if (c->struct_size != sizeof(cs_moe_config)) return invalid(who, "config.struct_size mismatch");
  if (c->format != CS_WEIGHTS_E2M1 && c->format != CS_WEIGHTS_BF16) return invalid(who, "format");
  if (c->hidden <= 0 || c->inter <= 0 || c->n_experts <= 0 || c->n_shared < 0 || c->top <= 0 || c->top > c->n_experts) return invalid(who, "sizes");
  if (c->hidden % 32 || c->inter % 32 || c->hidden > 65536 || c->inter > 65536)
    return unsupported(who, "hidden and inter must be multiples of 32, at most 65536");
  if (c->n_experts > MAX_EXPERTS || c->top > MAX_TOP || (int64_t)c->top + c->n_shared > 64)
    return unsupported(who, "at most 1024 experts, 32 of them a row, and 64 with the shared ones");
  if (c->score != CS_SCORE_SOFTMAX && c->score != CS_SCORE_SIGMOID) return invalid(who, "score");
  if (!is_flag(c->renormalise)) return invalid(who, "renormalise must be 0 or 1");
  if (!(c->scale - c->scale == 0)) return invalid(who, "scale must be finite");
  if (cs_status st = check_n_rows(who, n_rows)) return st;
  a.n_rows = n_rows;
  a.hidden = c->hidden; a.inter = c->inter; a.experts = c->n_experts; a.shared = c->n_shared; a.top = c->top;
  a.sigmoid = c->score == CS_SCORE_SIGMOID; a.renormalise = c->renormalise; a.scale = c->scale;
  const int64_t matrices = (int64_t)c->n_experts + c->n_shared;
  a.up_shape = packed_shape(c->format, matrices, 2 * c->inter, c->hidden);
  a.down_shape = packed_shape(c->format, matrices, c->hidden, c->inter);
  return CS_OK;
}

cs_status moe(const cs_moe_config* c, const void* x, int64_t x_row, const void* router, const float* choice_bias, const uint8_t* live,
              const void* up, const void* down, void* y, int64_t y_row, int32_t* experts, float* weights, int64_t n_rows, void* workspace,
              size_t workspace_bytes, void* stream) {
  const char* who = "cs_moe";
  MoeArgs a = {};
  if (cs_status st = moe_args(who, c, n_rows, a)) return st;
  if (n_rows == 0) return CS_OK;
  if (cs_status st = check_rows(who, "x", x, x_row, c->hidden, 2)) return st;
  if (n_rows > 1 && x_row > 1 << 17) return unsupported(who, "rows of x at most 2^17 elements apart");
  if (cs_status st = check_rows(who, "y", y, y_row, c->hidden, 2)) return st;
  if (!router || !aligned(router, 16) || !up || !aligned(up, 16) || !down || !aligned(down, 16)) return invalid(who, "NULL or misaligned weights");
  if (!experts || !aligned(experts, 4) || !weights || !aligned(weights, 4) || !aligned(choice_bias, 4))
    return invalid(who, "NULL or misaligned experts, weights or bias");
  if (cs_status st = check_workspace(who, workspace, workspace_bytes, moe_workspace(a))) return st;
  a.x = static_cast<const bf16_t*>(x); a.x_row = x_row;
  a.router = static_cast<const bf16_t*>(router); a.choice_bias = choice_bias; a.live = live;
  a.up = static_cast<const unsigned char*>(up); a.down = static_cast<const unsigned char*>(down);
  a.y = static_cast<bf16_t*>(y); a.y_row = y_row;
  a.experts_out = experts; a.weights_out = weights;
  return launch_moe(a, workspace, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

cs_status cs_norm_residual(const cs_norm_config* config, const void* x, int64_t x_row, const void* residual, int64_t residual_row,
                           const void* gate, int64_t gate_row, const float* post_gain, const float* post_bias, const float* pre_gain,
                           const float* pre_bias, void* r, int64_t r_row, void* y, int64_t y_row, int64_t n_rows, void* stream) try {
  return norm_residual(config, x, x_row, residual, residual_row, gate, gate_row, post_gain, post_bias, pre_gain, pre_bias, r, r_row, y, y_row,
                       n_rows, stream);
}
CS_CATCH_ALL("cs_norm_residual")

cs_status cs_weights_query(const cs_weights_config* config, size_t* bytes) try {
  PackedShape shape;
  if (!bytes) return invalid("cs_weights_query", "NULL argument");
  if (cs_status st = check_weights("cs_weights_query", config, shape)) return st;
  *bytes = (size_t)(shape.matrices * matrix_bytes(shape));
  return CS_OK;
}
CS_CATCH_ALL("cs_weights_query")

cs_status cs_weights_pack(const cs_weights_config* config, const void* w, int64_t w_row, int64_t w_matrix, int32_t dtype, void* packed,
                          int32_t* err_flag, void* stream) try {
  PackArgs a = {};
  if (cs_status st = weights("cs_weights_pack", config, w, w_row, w_matrix, dtype, packed, err_flag, a)) return st;
  return launch_weights_pack(a, dtype, static_cast<hipStream_t>(stream));
}
CS_CATCH_ALL("cs_weights_pack")

cs_status cs_weights_read(const cs_weights_config* config, const void* packed, void* w, int64_t w_row, int64_t w_matrix, int32_t dtype,
                          void* stream) try {
  PackArgs a = {};
  if (cs_status st = weights("cs_weights_read", config, w, w_row, w_matrix, dtype, packed, nullptr, a)) return st;
  // (the last row's place in 128 bits: 2^24 rows of 2^40 values pass 64)
  if (config->matrices > 1 && w_matrix < (__int128)(config->n - 1) * w_row + config->k) return invalid("cs_weights_read", "matrices overlap");
  return launch_weights_read(a, dtype, static_cast<hipStream_t>(stream));
}
CS_CATCH_ALL("cs_weights_read")

cs_status cs_linear_packed_query(const cs_weights_config* config, int64_t n_rows, size_t* workspace_bytes) try {
  LinearArgs a = {};
  if (!workspace_bytes) return invalid("cs_linear_packed_query", "NULL argument");
  return linear_args("cs_linear_packed_query", config, n_rows, a, *workspace_bytes);
}
CS_CATCH_ALL("cs_linear_packed_query")

cs_status cs_linear_packed(const cs_weights_config* config, const void* packed, const void* x, int64_t x_row, const float* bias, void* out,
                           int64_t out_row, int32_t out_dtype, int64_t n_rows, void* workspace, size_t workspace_bytes, void* stream) try {
  return linear_packed(config, packed, x, x_row, bias, out, out_row, out_dtype, n_rows, workspace, workspace_bytes, stream);
}
CS_CATCH_ALL("cs_linear_packed")

cs_status cs_moe_query(const cs_moe_config* config, int64_t n_rows, size_t* workspace_bytes) try {
  MoeArgs a = {};
  if (!workspace_bytes) return invalid("cs_moe_query", "NULL argument");
  if (cs_status st = moe_args("cs_moe_query", config, n_rows, a)) return st;
  *workspace_bytes = n_rows ? moe_workspace(a) : 0;
  return CS_OK;
}
CS_CATCH_ALL("cs_moe_query")

cs_status cs_moe(const cs_moe_config* config, const void* x, int64_t x_row, const void* router, const float* choice_bias,
                 const uint8_t* live, const void* up, const void* down, void* y, int64_t y_row, int32_t* experts, float* weights,
                 int64_t n_rows, void* workspace, size_t workspace_bytes, void* stream) try {
  return moe(config, x, x_row, router, choice_bias, live, up, down, y, y_row, experts, weights, n_rows, workspace, workspace_bytes, stream);
}
CS_CATCH_ALL("cs_moe")

}  // extern "C"
