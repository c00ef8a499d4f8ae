// sls_attention_status over status words in host memory: lines of "prefill decode" on stdin,
// the two readings that follow and what the words hold then on stdout.
#include <cstdio>

#include "../../paper_2607_19368_gb300/csrc/attention_api.cu"

static int words[2];

namespace sls {
int prefill_status_word(int** w) { return *w = &words[0], SLS_OK; }
int decode_status_word(int** w) { return *w = &words[1], SLS_OK; }
int launch_qkv_append(const AppendArgs&, int, cudaStream_t) { return SLS_OK; }
size_t attention_prefill_workspace(const CacheView&, int64_t, int) { return 0; }
int launch_attention_prefill(const AttnArgs&, int, void*, cudaStream_t) { return SLS_OK; }
size_t attention_decode_workspace(const CacheView&, int) { return 0; }
int launch_attention_decode(const AttnArgs&, int, void*, cudaStream_t) { return SLS_OK; }
}  // namespace sls

extern "C" int sls_workspace_status(void* word, void*) {
  const int st = *(int*)word;
  *(int*)word = 0;
  return st;
}

int main() {
  while (std::scanf("%d %d", &words[0], &words[1]) == 2) {
    const int first = sls_attention_status(nullptr), left = words[0] + words[1];
    std::printf("%d %d %d\n", first, left, sls_attention_status(nullptr));
  }
  return 0;
}
