// More checks of the host side of the 4-bit products and of the norm, on the runtime
// and the stand-ins of ops4_host.cpp.
//
//   ops4_host_edges NAME     runs one check; exit code 0 if it holds
#define main checks_of_ops4_host
#include "ops4_host.cpp"
#undef main

namespace {

// Without k there is nothing to scale: the kernel is given no scales.
void no_k_no_scales() {
  Host u;
  CHECK(peat_matmul_f4(&u.h, PEAT_NVFP4, nullptr, 0, nullptr, u.floats(), nullptr, 0, nullptr, u.floats(), u.floats(), 3, 5, 0,
                       u.data(), 5, PEAT_F32, nullptr) == PEAT_OK);
  CHECK(rt.launches == 1 && rt.product.K == 0 && !rt.product.sa && !rt.product.sb && rt.product.bias == u.floats());
}

// A norm's rows of nothing: every output that has elements is written.
void norm_of_nothing() {
  Host u;
  float *scale = u.floats(), *rstd = u.floats() + 64;
  for (int i = 0; i < 4; i++) scale[i] = rstd[i] = 5.0f;
  auto run = [&](float* s, float* r, int8_t* q) {
    return peat_rmsnorm(&u.h, nullptr, 0, nullptr, 0, nullptr, PEAT_F32, 3, 0, PEAT_BF16, 1e-6f, nullptr, 0, nullptr, 0, q, 0, s,
                        nullptr, 0, r, nullptr);
  };
  CHECK(run(scale, rstd, nullptr) == PEAT_OK && rt.launches == 0);
  for (int i = 0; i < 3; i++) CHECK(scale[i] == 0.0f && rstd[i] != rstd[i]);
  CHECK(scale[3] == 5.0f && rstd[3] == 5.0f);
  CHECK(run(nullptr, nullptr, reinterpret_cast<int8_t*>(u.data())) == PEAT_OK && rt.launches == 0);
  CHECK(run(nullptr, nullptr, nullptr) == PEAT_OK && rt.launches == 0);  // (matrices of nothing may be NULL)
}

// The format that has no float32 scales takes none, here as in the other calls.
void mxfp4_has_no_scales() {
  Host u;
  auto run = [&](peat_f4_t format, const float* sa, const float* sb) {
    u.h.err.clear();
    return peat_matmul_f4(&u.h, format, u.bytes(), 64, u.bytes(), sa, u.bytes(), 64, u.bytes(), sb, nullptr, 5, 7, 128, u.data(), 7,
                          PEAT_F32, nullptr);
  };
  CHECK(run(PEAT_MXFP4, u.floats(), nullptr) == PEAT_ERR_INVALID_ARG && !u.h.err.empty());
  CHECK(run(PEAT_MXFP4, nullptr, u.floats()) == PEAT_ERR_INVALID_ARG && !u.h.err.empty());
  CHECK(rt.launches == 0);
  CHECK(run(PEAT_MXFP4, nullptr, nullptr) == PEAT_OK && run(PEAT_NVFP4, u.floats(), nullptr) == PEAT_OK && rt.launches == 2);
}

// What a product takes of the workspace is what the header says.
void workspace() {
  for (int format : {PEAT_MXFP4, PEAT_NVFP4})
    for (int axes = 0; axes < 4; axes++)
      for (int64_t K : {1, 16, 32, 33, 1000})
        for (int64_t rows : {1, 3, 128, 129, 1000}) {
          Host u;
          auto up = [](int64_t n, int64_t to) { return (n + to - 1) / to * to; };
          const int64_t R[2] = {rows, 77}, block = format == PEAT_MXFP4 ? 32 : 16;
          int64_t held = 0, tops = 0;
          peat_operand_f4_t op[2];
          for (int i = 0; i < 2; i++) {
            const bool down = axes >> i & 1;
            op[i] = peat_operand_f4_t{u.data(), nullptr, nullptr, down ? K : R[i], down ? R[i] : K, down ? R[i] : K, PEAT_BF16, down};
            held += up(R[i] * up(up(K, block) / 2, 16), 256) + up(peat_f4_scale_bytes(R[i], up(K, block) / block), 256);
            if (format == PEAT_NVFP4) held += up(4 * R[i], 256);
            if (format == PEAT_NVFP4 && down) tops += 128 * R[i];
          }
          CHECK(peat_product_f4(&u.h, (peat_f4_t)format, &op[0], &op[1], nullptr, u.data(), 77, PEAT_F32, nullptr) == PEAT_OK);
          CHECK((int64_t)u.h.ops->rounded_cap == held && (int64_t)u.h.ops->tops_cap == tops);
        }
}

}  // namespace

int main(int argc, char** argv) {
  const std::map<std::string, void (*)()> checks = {{"no_k_no_scales", no_k_no_scales}, {"norm_of_nothing", norm_of_nothing},
                                                    {"mxfp4_has_no_scales", mxfp4_has_no_scales},
                                                    {"workspace", workspace}};
  if (argc != 2 || !checks.count(argv[1])) return 2;
  checks.at(argv[1])();
  return failures ? 1 : 0;
}
