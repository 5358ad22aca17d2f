// octo_op_product: arguments, their checks and the choice of a kernel.
#include "product.h"

using namespace octo;

namespace {
bool rows_near(long long bytes) { return bytes >= 0 && bytes <= 8 << 20; }        // 255 of them stay within 31 bits
constexpr int MOST_K = 1 << 30;                                                   // bytes of a row: with 63 rows before it, where they are loaded from one address, within 31 bits
}  // namespace

extern "C" octo_status octo_op_product(const octo_product_op* op, void* hip_stream, int32_t* kernel_id) {
  if (kernel_id) *kernel_id = 0;
  if (!op || (op->dtype != OCTO_F32 && op->dtype != OCTO_F16 && op->dtype != OCTO_BF16)) return OCTO_EINVAL;
  if (op->x_format < OCTO_ROWS_PLAIN || op->x_format > OCTO_ROWS_MX8 || op->y_format < OCTO_ROWS_PLAIN || op->y_format > OCTO_ROWS_MX8) return OCTO_EINVAL;
  if (op->n < 0 || op->k < 1 || op->cols < 1 || op->cols > 0x20000000 || op->act < OCTO_ACT_NONE || op->act > OCTO_ACT_GELU) return OCTO_EINVAL;
  const bool x8 = op->x_format == OCTO_ROWS_MX8, y8 = op->y_format == OCTO_ROWS_MX8;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  ProductArgs a{};
  if (x8) {
    if (op->k % 32 || op->k > MOST_K || !mx8_ok(op->x8) || !mx8_ok(op->w8) || op->x8.exp_row > 8 << 20 || op->w8.exp_row > 8 << 20) return OCTO_EINVAL;
    a.x = (const char*)op->x8.d_codes; a.w = (const char*)op->w8.d_codes; a.x_row = op->x8.code_row; a.w_row = op->w8.code_row;
    a.xe = op->x8.d_exps; a.we = op->w8.d_exps; a.xe_row = op->x8.exp_row; a.we_row = op->w8.exp_row;
    a.k_bytes = op->k;
    a.exp_words = op->k % 128 == 0 && !(((uintptr_t)a.xe | (uintptr_t)a.we | (uintptr_t)a.xe_row | (uintptr_t)a.we_row) & 3);
  } else {
    if (!op->d_x || !op->d_w || (((uintptr_t)op->d_x | (uintptr_t)op->d_w) & 15) || op->k > MOST_K / es || op->k * es % 16) return OCTO_EINVAL;
    if (op->x_row < 0 || op->w_row < 0 || op->x_row > 8 << 20 || op->w_row > 8 << 20 || (op->x_row * es & 15) || (op->w_row * es & 15)) return OCTO_EINVAL;
    a.x = (const char*)op->d_x; a.w = (const char*)op->d_w; a.x_row = op->x_row * es; a.w_row = op->w_row * es;
    a.k_bytes = op->k * es;
  }
  if (!rows_near(a.x_row) || !rows_near(a.w_row)) return OCTO_EINVAL;
  const int ys = op->out_f32 ? 4 : es;
  if (y8) {
    if (op->out_f32 || op->d_res || op->cols % 32 || !mx8_ok(op->y8)) return OCTO_EINVAL;
  } else if (!op->d_y || op->y_row < 0 || ((uintptr_t)op->d_y | (uintptr_t)op->d_res) % ys || (op->d_res && op->res_row < 0)) {
    return OCTO_EINVAL;
  }
  if (((uintptr_t)op->d_bias & 3) || ((uintptr_t)op->d_n & 3)) return OCTO_EINVAL;
  a.bias = op->d_bias; a.res = op->d_res; a.y = op->d_y; a.res_row = op->res_row; a.y_row = op->y_row; a.y8 = op->y8;
  a.n_dyn = op->d_n; a.n = op->n; a.cols = op->cols; a.gated = op->gated != 0; a.act = op->act;
  a.y_kind = y8 ? PRODUCT_Y_MX8 : op->out_f32 || op->dtype == OCTO_F32 ? PRODUCT_Y_F32 : op->dtype == OCTO_F16 ? PRODUCT_Y_F16 : PRODUCT_Y_BF16;
  a.y_vec = !((uintptr_t)op->d_y % (4 * ys)) && op->y_row % 4 == 0;
  a.res_vec = !((uintptr_t)op->d_res % (4 * ys)) && op->res_row % 4 == 0;
  a.bias_vec = !((uintptr_t)op->d_bias & 15) && (!a.gated || op->cols % 4 == 0);
  const uintptr_t at = (uintptr_t)op->d_y | (uintptr_t)op->d_res;
  a.direct = op->act != OCTO_ACT_GELU && (!a.bias || a.bias_vec) && (y8 || (ys == 2 && !(at & 15) && op->cols % 8 == 0 && op->y_row % 8 == 0 && (!a.res || op->res_row % 8 == 0)));
  a.vec = !y8 && a.cols % 4 == 0 && a.y_vec && (!a.res || a.res_vec) && (!a.bias || a.bias_vec);
  a.exact8 = x8 && (!op->fast8 || a.y_kind == PRODUCT_Y_F32 || !a.exp_words);
  if (!op->n) return OCTO_OK;
  hipStream_t s = (hipStream_t)hip_stream;
  const int bits = x8 ? 8 : 8 * es;
  auto choice = [&](int n) { return product_choice(n, a.k_bytes, a.cols, a.gated, y8, bits, !x8 || a.exp_words, x8 && !a.exp_words, a.direct); };
  const ProductChoice first = choice(op->n);
  if (first.blocks > 0x7FFFFF) return OCTO_EINVAL;                   // HIP counts the threads of a launch, up to 512 a block, in 32 bits
  for (ProductChoice c = first;;) {
    a.n = c.tokens;
    const hipError_t e = x8 ? launch_product<f8>(c.variant, a, s) : op->dtype == OCTO_F32 ? launch_product<float>(c.variant, a, s)
                       : op->dtype == OCTO_F16 ? launch_product<_Float16>(c.variant, a, s) : launch_product<__bf16>(c.variant, a, s);
    if (e != hipSuccess) return OCTO_EHIP;
    const long long m = c.tokens;
    a.n_from += c.tokens;
    if (a.n_from >= op->n) break;
    a.x += m * a.x_row;
    if (x8) a.xe += m * a.xe_row;
    if (a.res) a.res = (const char*)a.res + m * a.res_row * ys;
    if (y8) { a.y8.d_codes += m * a.y8.code_row; a.y8.d_exps += m * a.y8.exp_row; }
    else a.y = (char*)a.y + m * a.y_row * ys;
    c = choice(op->n - a.n_from);
  }
  if (kernel_id) *kernel_id = first.variant;
  return OCTO_OK;
}
