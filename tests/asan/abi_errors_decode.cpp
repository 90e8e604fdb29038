// Host-side argument checks of the entry points for rotary positions, log
// probabilities and attention with sinks or shared prefixes, for a build of
// the library's host code under AddressSanitizer.  Every call below is rejected
// on the host before any HIP call: the pointers are fake, aligned addresses that
// are never dereferenced, so this program must run where no GPU is visible.
// Exit status 0 when every call returns the expected status.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "tq.h"

namespace {

int failures = 0;

void expect(const char* what, int got, int want) {
  if (got != want) {
    std::printf("FAIL %s: got %d, want %d\n", what, got, want);
    ++failures;
  }
}

const uintptr_t kFake = 0x7F0000000000ull;   // 256-byte aligned, never dereferenced
template <class T>
T* fake(uintptr_t off = 0) {
  return reinterpret_cast<T*>(kFake + off);
}

tq_kv_cache cache() {
  tq_kv_cache c;
  std::memset(&c, 0, sizeof c);
  c.n_layers = 2;
  c.n_kv_heads = 4;
  c.head_dim = 128;
  c.group = 64;
  c.page_size = 64;
  c.n_seqs = 8;
  c.max_pages = 1000;
  c.n_pages = 4000;
  c.data = fake<uint8_t>();
  c.pages = fake<int32_t>(0x100000);
  c.lens = fake<int32_t>(0x200000);
  c.refs = fake<int32_t>(0x300000);
  return c;
}

tq_kv_attn attn() {
  tq_kv_attn a;
  std::memset(&a, 0, sizeof a);
  a.n_rows = 8;
  a.n_tokens = 8;
  a.max_q = 1;
  a.n_heads = 16;
  a.scale = 0.1f;
  a.q.data = fake<const uint16_t>();
  a.q.token_stride = 16 * 128;
  a.q.head_stride = 128;
  a.o = fake<void>();
  a.workspace = fake<void>();
  a.workspace_bytes = (size_t)1 << 40;
  return a;
}

tq_kv_scope scope() {
  tq_kv_scope s;
  std::memset(&s, 0, sizeof s);
  s.n_groups = 1;
  s.prefix = fake<const int32_t>();
  return s;
}

tq_rope_call rope() {
  tq_rope_call c;
  std::memset(&c, 0, sizeof c);
  c.n_tokens = 3;
  c.n_heads = 4;
  c.n_kv_heads = 2;
  c.head_dim = 128;
  c.rot = 96;
  c.n_axes = 3;
  c.scale = 1.0f;
  c.positions = fake<const int32_t>();
  c.axis_stride = 3;
  c.freq = fake<const float>(0x1000);
  c.axis = fake<const uint8_t>(0x2000);
  c.q = tq_kv_rows{fake<const uint16_t>(0x10000), 512, 128};
  c.k = tq_kv_rows{fake<const uint16_t>(0x20000), 256, 128};
  c.q_out = tq_out_rows{fake<uint16_t>(0x30000), 512, 128};
  c.k_out = tq_out_rows{fake<uint16_t>(0x40000), 256, 128};
  return c;
}

tq_logprobs_call logprobs() {
  tq_logprobs_call c;
  std::memset(&c, 0, sizeof c);
  c.n_rows = 2;
  c.n_vocab = 50000;
  c.n_ids = 3;
  c.n_top = 5;
  c.flags = TQ_LOGITS_FP16;
  c.scale = 1.0f;
  c.logits = fake<const void>();
  c.ld = 50000;
  c.ids = fake<const int32_t>(0x100000);
  c.logp = fake<float>(0x200000);
  c.entropy = fake<float>(0x300000);
  c.top_ids = fake<int32_t>(0x400000);
  c.top_logp = fake<float>(0x500000);
  c.d_err = fake<int32_t>(0x600000);
  c.workspace = fake<void>(0x700000);
  c.workspace_bytes = (size_t)1 << 40;
  return c;
}

tq_status attend(const tq_kv_attn& a, const tq_kv_scope& s) {
  const tq_kv_cache c = cache();
  return tq_kv_attention_scope(&c, 0, &a, &s, nullptr);
}

}  // namespace

int main() {
  {   // attention's own arguments
    const tq_kv_cache good = cache();
    tq_kv_attn a = attn();
    tq_kv_scope s = scope();
    expect("cache", tq_kv_attention_scope(nullptr, 0, &a, &s, nullptr), TQ_ERR_NULL);
    expect("call", tq_kv_attention_scope(&good, 0, nullptr, &s, nullptr), TQ_ERR_NULL);
    expect("scope", tq_kv_attention_scope(&good, 0, &a, nullptr, nullptr), TQ_ERR_NULL);
    expect("layer", tq_kv_attention_scope(&good, 2, &a, &s, nullptr), TQ_ERR_SHAPE);
    expect("layer < 0", tq_kv_attention_scope(&good, -1, &a, &s, nullptr), TQ_ERR_SHAPE);
    a = attn(); a.n_heads = 15; expect("heads", attend(a, s), TQ_ERR_SHAPE);
    a = attn(); a.window = -1; expect("window", attend(a, s), TQ_ERR_SHAPE);
    a = attn(); a.scale = INFINITY; expect("scale", attend(a, s), TQ_ERR_SHAPE);
    a = attn(); a.flags = 2; expect("flags", attend(a, s), TQ_ERR_UNSUPPORTED);
    a = attn(); a.q.data = nullptr; expect("q", attend(a, s), TQ_ERR_NULL);
    a = attn(); a.o = nullptr; expect("o", attend(a, s), TQ_ERR_NULL);
    a = attn(); a.o = fake<void>(8); expect("o align", attend(a, s), TQ_ERR_ALIGN);
    a = attn(); a.lse = fake<float>(2); expect("lse align", attend(a, s), TQ_ERR_ALIGN);
    a = attn(); a.seqs = fake<const int32_t>(2); expect("seqs align", attend(a, s), TQ_ERR_ALIGN);
    a = attn(); a.cu_q = fake<const int32_t>(2); expect("cu_q align", attend(a, s), TQ_ERR_ALIGN);
  }
  {   // the scope
    const tq_kv_attn a = attn();
    tq_kv_scope s;
    s = scope(); s.sinks = -1; expect("sinks", attend(a, s), TQ_ERR_SHAPE);
    s = scope(); s.n_groups = -1; expect("groups < 0", attend(a, s), TQ_ERR_SHAPE);
    s = scope(); s.n_groups = 9; s.cu_rows = fake<const int32_t>(); expect("groups > rows", attend(a, s), TQ_ERR_SHAPE);
    s = scope(); s.n_groups = 2; expect("two groups without cu_rows", attend(a, s), TQ_ERR_SHAPE);
    s = scope(); s.max_prefix = -1; expect("max_prefix", attend(a, s), TQ_ERR_SHAPE);
    s = scope(); s.max_tail = -1; expect("max_tail", attend(a, s), TQ_ERR_SHAPE);
    s = scope(); s.prefix = nullptr; expect("prefix", attend(a, s), TQ_ERR_NULL);
    s = scope(); s.prefix = fake<const int32_t>(2); expect("prefix align", attend(a, s), TQ_ERR_ALIGN);
    s = scope(); s.cu_rows = fake<const int32_t>(2); expect("cu_rows align", attend(a, s), TQ_ERR_ALIGN);
  }
  for (int shared = 0; shared < 2; ++shared) {   // workspaces: of sinks beside a window, of a shared prefix
    const tq_kv_cache good = cache();
    tq_kv_attn a = attn();
    tq_kv_scope s = scope();
    if (!shared) {
      s.n_groups = 0;
      s.sinks = 4;
      a.n_rows = a.n_tokens = 1;
      a.window = 20000;
    } else {
      s.max_prefix = 60000;
      s.max_tail = 100;
    }
    const size_t need = tq_kv_attention_scope_workspace_bytes(&good, &a, &s);
    expect("needs a workspace", need > TQ_WORKSPACE_COUNT_BYTES, 1);
    tq_kv_attn b = a;
    b.workspace = nullptr; expect("workspace", attend(b, s), TQ_ERR_NULL);
    b = a; b.workspace_bytes = need - 1; expect("workspace size", attend(b, s), TQ_ERR_SHAPE);
    b = a; b.workspace = fake<void>(8); expect("workspace align", attend(b, s), TQ_ERR_ALIGN);
    b = a; b.n_rows = 0; expect("workspace of bad arguments",
                                (int)tq_kv_attention_scope_workspace_bytes(&good, &b, &s), 0);
    s.sinks = -1; expect("workspace of a bad scope", (int)tq_kv_attention_scope_workspace_bytes(&good, &a, &s), 0);
  }
  {   // more tiles than a launch takes
    tq_kv_cache c = cache();
    c.n_kv_heads = 1024;
    tq_kv_attn a = attn();
    a.n_heads = 1024; a.n_rows = 1; a.n_tokens = a.max_q = 1 << 20;
    tq_kv_scope s = scope();
    expect("tiles", tq_kv_attention_scope(&c, 0, &a, &s, nullptr), TQ_ERR_UNSUPPORTED);
  }
  {   // shared prefixes
    const tq_kv_cache good = cache();
    int32_t* p = fake<int32_t>();
    const int32_t* cu = fake<const int32_t>(0x1000);
    expect("prefix: cache", tq_kv_shared_prefix(nullptr, nullptr, cu, 2, 8, p, nullptr), TQ_ERR_NULL);
    tq_kv_cache c = cache();
    c.page_size = 48; expect("prefix: page size", tq_kv_shared_prefix(&c, nullptr, cu, 2, 8, p, nullptr) != TQ_OK, 1);
    expect("prefix: rows", tq_kv_shared_prefix(&good, nullptr, cu, 1, 0, p, nullptr), TQ_ERR_SHAPE);
    expect("prefix: rows without seqs", tq_kv_shared_prefix(&good, nullptr, cu, 2, 9, p, nullptr), TQ_ERR_SHAPE);
    expect("prefix: no groups", tq_kv_shared_prefix(&good, nullptr, cu, 0, 8, p, nullptr), TQ_ERR_SHAPE);
    expect("prefix: groups > rows", tq_kv_shared_prefix(&good, nullptr, cu, 9, 8, p, nullptr), TQ_ERR_SHAPE);
    expect("prefix: groups without cu", tq_kv_shared_prefix(&good, nullptr, nullptr, 2, 8, p, nullptr), TQ_ERR_SHAPE);
    expect("prefix: output", tq_kv_shared_prefix(&good, nullptr, cu, 2, 8, nullptr, nullptr), TQ_ERR_NULL);
    expect("prefix: output align", tq_kv_shared_prefix(&good, nullptr, cu, 2, 8, fake<int32_t>(2), nullptr), TQ_ERR_ALIGN);
    expect("prefix: cu align", tq_kv_shared_prefix(&good, nullptr, fake<const int32_t>(2), 2, 8, p, nullptr), TQ_ERR_ALIGN);
    expect("prefix: seqs align", tq_kv_shared_prefix(&good, fake<const int32_t>(2), cu, 2, 8, p, nullptr), TQ_ERR_ALIGN);
  }
  {   // rotary positions
    tq_rope_call c;
    auto run = [&] { return tq_rope(&c, nullptr); };
    expect("rope: call", tq_rope(nullptr, nullptr), TQ_ERR_NULL);
    c = rope(); c.n_tokens = 0; expect("rope: tokens", run(), TQ_ERR_SHAPE);
    c = rope(); c.n_tokens = TQ_ROPE_MAX_TOKENS + 1; expect("rope: most tokens", run(), TQ_ERR_UNSUPPORTED);
    c = rope(); c.n_heads = 0; expect("rope: heads", run(), TQ_ERR_SHAPE);
    c = rope(); c.n_heads = TQ_ROPE_MAX_HEADS + 1; expect("rope: most heads", run(), TQ_ERR_UNSUPPORTED);
    c = rope(); c.n_kv_heads = -1; expect("rope: kv heads", run(), TQ_ERR_SHAPE);
    c = rope(); c.n_kv_heads = TQ_ROPE_MAX_HEADS + 1; expect("rope: most kv heads", run(), TQ_ERR_UNSUPPORTED);
    c = rope(); c.rot = 0; expect("rope: rot", run(), TQ_ERR_SHAPE);
    c = rope(); c.rot = 95; expect("rope: odd rot", run(), TQ_ERR_SHAPE);
    c = rope(); c.rot = 130; expect("rope: rot > dim", run(), TQ_ERR_SHAPE);
    c = rope(); c.head_dim = TQ_ROPE_MAX_DIM + 2; expect("rope: dim", run(), TQ_ERR_UNSUPPORTED);
    c = rope(); c.n_axes = 0; expect("rope: axes", run(), TQ_ERR_SHAPE);
    c = rope(); c.n_axes = TQ_ROPE_MAX_AXES + 1; expect("rope: most axes", run(), TQ_ERR_UNSUPPORTED);
    c = rope(); c.flags = 4; expect("rope: flags", run(), TQ_ERR_UNSUPPORTED);
    c = rope(); c.scale = NAN; expect("rope: scale", run(), TQ_ERR_SHAPE);
    c = rope(); c.positions = nullptr; expect("rope: positions", run(), TQ_ERR_NULL);
    c = rope(); c.freq = nullptr; expect("rope: freq", run(), TQ_ERR_NULL);
    c = rope(); c.q.data = nullptr; expect("rope: q", run(), TQ_ERR_NULL);
    c = rope(); c.q_out.data = nullptr; expect("rope: q_out", run(), TQ_ERR_NULL);
    c = rope(); c.k.data = nullptr; expect("rope: k", run(), TQ_ERR_NULL);
    c = rope(); c.k_out.data = nullptr; expect("rope: k_out", run(), TQ_ERR_NULL);
    c = rope(); c.positions = fake<const int32_t>(2); expect("rope: positions align", run(), TQ_ERR_ALIGN);
    c = rope(); c.freq = fake<const float>(2); expect("rope: freq align", run(), TQ_ERR_ALIGN);
    c = rope(); c.q.data = fake<const uint16_t>(1); expect("rope: q align", run(), TQ_ERR_ALIGN);
    c = rope(); c.k_out.data = fake<uint16_t>(1); expect("rope: k_out align", run(), TQ_ERR_ALIGN);
    c = rope(); c.q_out.token_stride = 0; expect("rope: tokens on each other", run(), TQ_ERR_SHAPE);
    c = rope(); c.k_out.head_stride = 0; expect("rope: heads on each other", run(), TQ_ERR_SHAPE);
    c = rope(); c.q_out.data = fake<uint16_t>(0x10000); c.q_out.token_stride = 513;
    expect("rope: in place with other strides", run(), TQ_ERR_SHAPE);
    c = rope(); c.k_out.data = fake<uint16_t>(0x20000); c.k_out.head_stride = 130;
    expect("rope: keys in place with other strides", run(), TQ_ERR_SHAPE);
  }
  {   // log probabilities
    tq_logprobs_call c;
    auto run = [&] { return tq_logprobs(&c, nullptr); };
    expect("logprobs: call", tq_logprobs(nullptr, nullptr), TQ_ERR_NULL);
    expect("logprobs: workspace of nothing", (int)tq_logprobs_workspace_bytes(nullptr), 0);
    c = logprobs(); c.n_rows = 0; expect("logprobs: rows", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.n_rows = (1 << 20) + 1; expect("logprobs: most rows", run(), TQ_ERR_UNSUPPORTED);
    c = logprobs(); c.n_vocab = 0; expect("logprobs: vocabulary", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.ld = c.n_vocab = (1 << 24) + 1; expect("logprobs: most tokens", run(), TQ_ERR_UNSUPPORTED);
    c = logprobs(); c.ld = 49999; expect("logprobs: ld", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.n_ids = -1; expect("logprobs: ids < 0", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.n_ids = TQ_LOGPROBS_MAX_IDS + 1; expect("logprobs: most ids", run(), TQ_ERR_UNSUPPORTED);
    c = logprobs(); c.n_top = -1; expect("logprobs: top < 0", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.n_top = TQ_LOGPROBS_MAX_TOP + 1; expect("logprobs: most top", run(), TQ_ERR_UNSUPPORTED);
    c = logprobs(); c.n_vocab = 4; expect("logprobs: top > vocabulary", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.flags = 2; expect("logprobs: flags", run(), TQ_ERR_UNSUPPORTED);
    c = logprobs(); c.scale = 0.0f; expect("logprobs: scale 0", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.scale = NAN; expect("logprobs: scale NaN", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.scale = 2e18f; expect("logprobs: scale", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.logits = nullptr; expect("logprobs: logits", run(), TQ_ERR_NULL);
    c = logprobs(); c.ids = nullptr; expect("logprobs: ids", run(), TQ_ERR_NULL);
    c = logprobs(); c.logp = nullptr; expect("logprobs: logp", run(), TQ_ERR_NULL);
    c = logprobs(); c.top_ids = nullptr; expect("logprobs: top_ids", run(), TQ_ERR_NULL);
    c = logprobs(); c.top_logp = nullptr; expect("logprobs: top_logp", run(), TQ_ERR_NULL);
    c = logprobs(); c.logits = fake<const void>(1); expect("logprobs: logits align", run(), TQ_ERR_ALIGN);
    c = logprobs(); c.flags = TQ_LOGITS_FP32; c.logits = fake<const void>(2);
    expect("logprobs: fp32 logits align", run(), TQ_ERR_ALIGN);
    c = logprobs(); c.ids = fake<const int32_t>(2); expect("logprobs: ids align", run(), TQ_ERR_ALIGN);
    c = logprobs(); c.logp = fake<float>(2); expect("logprobs: logp align", run(), TQ_ERR_ALIGN);
    c = logprobs(); c.entropy = fake<float>(2); expect("logprobs: entropy align", run(), TQ_ERR_ALIGN);
    c = logprobs(); c.d_err = fake<int32_t>(2); expect("logprobs: d_err align", run(), TQ_ERR_ALIGN);
    c = logprobs();
    const size_t need = tq_logprobs_workspace_bytes(&c);
    expect("logprobs: few rows are cut in parts", need > TQ_WORKSPACE_COUNT_BYTES, 1);
    c.workspace = nullptr; expect("logprobs: workspace", run(), TQ_ERR_NULL);
    c = logprobs(); c.workspace_bytes = need - 1; expect("logprobs: workspace size", run(), TQ_ERR_SHAPE);
    c = logprobs(); c.workspace = fake<void>(8); expect("logprobs: workspace align", run(), TQ_ERR_ALIGN);
  }

  std::printf("%s: %d failure(s)\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
