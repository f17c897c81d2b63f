// elasto_op_residual_norm: which form of the kernel (residual_norm.cuh) a call gets, and the form for rows of whole eights.
#include "residual_norm.cuh"

namespace elasto {

cudaError_t residual_norm_launch(const elasto_residual_norm_args& u, int* status, cudaStream_t s) {
  // rows that start on multiples of eight values in memory, and tables that can be read 16 bytes at a time
  auto wide = [](const void* p, long long row, int type) {
    const int size = type == ELASTO_F32 ? 4 : type == ELASTO_E4M3 ? 1 : 2;
    return !p || (reinterpret_cast<uintptr_t>(p) % (8 * size) == 0 && row % 8 == 0);
  };
  bool vec = u.cols % 8 == 0 && wide(u.x, u.x_row, u.x_type) && wide(u.y, u.y_row, u.y_type) && wide(u.x_out, u.x_out_row, u.x_type) &&
             wide(u.z, u.z_row, u.z_type);
  for (const void* p : {u.gate, u.shift, u.scale}) vec = vec && (!p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && u.mod_row % 8 == 0));
  return vec ? residual::launch<true>(u, status, s) : residual_norm_any_launch(u, status, s);
}

}  // namespace elasto
