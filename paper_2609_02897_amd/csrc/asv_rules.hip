// The bf16 LM head with sampling rules: K1's kernels once more, with the rules behind the product (a
// translation unit of its own, as they take the longest to compile).
#include "asv_host.h"
#include "asv_k1_host.h"
#include "k_rules.h"

namespace asv {

int verify_bf16_ruled(const asv_verify_args* a, char* ws, const RuleArgs& r, hipStream_t s) {
  return verify_bf16(a, ws, nullptr, nullptr, nullptr, s, r);
}

}  // namespace asv
