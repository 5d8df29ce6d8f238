// What a context keeps for the attention calls (lv_kv.cu), whose translation
// unit does not see the rest of it.
#pragma once

#include <cstddef>

#include "llmvisor.h"

namespace lv {

struct KvHost {
  int sms = 0;
  int *d_status = nullptr;           // the context's status word
  unsigned char *scratch = nullptr;  // owned
  size_t cap = 0;
  void *outgrown[64] = {};           // owned: earlier scratch, which captured calls may still use
  int n_outgrown = 0;
  unsigned configured = 0;           // kernels whose shared-memory limit is set, a bit each
  unsigned long long *counter = nullptr;  // owned: two counters of work that kernels hand out, zero between calls
};

KvHost *kv_host(lv_ctx *ctx);

}  // namespace lv
