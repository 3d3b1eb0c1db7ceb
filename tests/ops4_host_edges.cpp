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

}  // namespace

int main(int argc, char** argv) {
  const std::map<std::string, void (*)()> checks = {{"no_k_no_scales", no_k_no_scales}};
  if (argc != 2 || !checks.count(argv[1])) return 2;
  checks.at(argv[1])();
  return failures ? 1 : 0;
}
