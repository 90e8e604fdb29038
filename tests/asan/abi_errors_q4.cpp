// Host-side argument checks of the 4-bit entry points of include/tq.h, for a
// build of the library's host code under AddressSanitizer.  Every call below
// is rejected on the host before any HIP call: the pointers are fake, aligned
// addresses that are never dereferenced, so this program must run where no
// GPU is visible.  Exit status 0 when every call returns the expected status.
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

tq_q4_matrix mat() {
  tq_q4_matrix m;
  std::memset(&m, 0, sizeof m);
  m.n_out = 33;
  m.n_in = 300;
  m.group = 64;
  m.codes = fake<const uint8_t>();
  m.params = fake<const uint16_t>(0x100000);
  return m;
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
  c.max_pages = 16;
  c.n_pages = 100;
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

int extend(const tq_kv_cache& c, int n = 8, const int32_t* seqs = nullptr, int32_t* starts = fake<int32_t>()) {
  return tq_kv_extend(&c, seqs, nullptr, n, starts, nullptr, nullptr);
}

int attend(const tq_kv_cache& c, const tq_kv_attn& a, int layer = 0) { return tq_kv_attention(&c, layer, &a, nullptr); }

}  // namespace

int main() {
  {
    expect("code bytes", (int)tq_q4_code_bytes(33, 300), 3 * 3 * 1024);
    expect("param bytes", (int)tq_q4_param_bytes(33, 300, 64), 3 * 6 * 64);
    expect("code bytes of nothing", (int)tq_q4_code_bytes(0, 300), 0);
    expect("code bytes past the tiles", (int)tq_q4_code_bytes(TQ_Q4_MAX_OUT, TQ_Q4_MAX_IN), 0);
    expect("param bytes of group 16", (int)tq_q4_param_bytes(33, 300, 16), 0);
    const uint16_t* X = fake<const uint16_t>();
    auto gemm = [&](const tq_q4_matrix& m, const uint16_t* x, int64_t ldx, int B, void* y, int flags) {
      return (int)tq_q4_gemm(&m, x, ldx, B, y, flags, nullptr, 0, nullptr);
    };
    void* Y = fake<void>();
    tq_q4_matrix m = mat();
    m.group = 48; expect("q4 group", gemm(m, X, 300, 1, Y, 0), TQ_ERR_UNSUPPORTED);
    m = mat(); m.reserved = 1; expect("q4 reserved", gemm(m, X, 300, 1, Y, 0), TQ_ERR_SHAPE);
    m = mat(); m.n_out = 0; expect("q4 n_out", gemm(m, X, 300, 1, Y, 0), TQ_ERR_SHAPE);
    m = mat(); m.n_in = -1; expect("q4 n_in", gemm(m, X, 300, 1, Y, 0), TQ_ERR_SHAPE);
    m = mat(); m.n_in = TQ_Q4_MAX_IN + 1; expect("q4 n_in limit", gemm(m, X, 1 << 30, 1, Y, 0), TQ_ERR_UNSUPPORTED);
    m = mat(); m.n_out = TQ_Q4_MAX_OUT; m.n_in = 65536; expect("q4 tiles", gemm(m, X, 65536, 1, Y, 0), TQ_ERR_UNSUPPORTED);
    m = mat(); m.codes = nullptr; expect("q4 codes", gemm(m, X, 300, 1, Y, 0), TQ_ERR_NULL);
    m = mat(); m.params = fake<const uint16_t>(8); expect("q4 params align", gemm(m, X, 300, 1, Y, 0), TQ_ERR_ALIGN);
    m = mat();
    expect("q4 X", gemm(m, nullptr, 300, 1, Y, 0), TQ_ERR_NULL);
    expect("q4 Y", gemm(m, X, 300, 1, nullptr, 0), TQ_ERR_NULL);
    expect("q4 ldx", gemm(m, X, 299, 1, Y, 0), TQ_ERR_SHAPE);
    expect("q4 batch 0", gemm(m, X, 300, 0, Y, 0), TQ_ERR_SHAPE);
    expect("q4 batch 65", gemm(m, X, 300, 65, Y, 0), TQ_ERR_SHAPE);
    expect("q4 flags", gemm(m, X, 300, 1, Y, 2), TQ_ERR_UNSUPPORTED);
    expect("q4 X align", gemm(m, reinterpret_cast<const uint16_t*>(kFake + 1), 300, 1, Y, 0), TQ_ERR_ALIGN);
    expect("q4 Y align", gemm(m, X, 300, 1, fake<void>(2), 0), TQ_ERR_ALIGN);
    expect("q4 matrix", tq_q4_gemm(nullptr, X, 300, 1, Y, 0, nullptr, 0, nullptr), TQ_ERR_NULL);
    {
      tq_q4_matrix deep = mat();
      deep.n_in = 4096;
      const size_t need = tq_q4_workspace_bytes(&deep, 64);
      expect("q4 workspace", need > 0, 1);
      expect("q4 workspace of few rows", (int)tq_q4_workspace_bytes(&deep, 16), 0);
      expect("q4 workspace of 65 rows", (int)tq_q4_workspace_bytes(&deep, 65), 0);
      expect("q4 workspace size", tq_q4_gemm(&deep, X, 4096, 64, Y, 0, fake<void>(), need - 1, nullptr), TQ_ERR_SHAPE);
      expect("q4 workspace align", tq_q4_gemm(&deep, X, 4096, 64, Y, 0, fake<void>(8), need, nullptr), TQ_ERR_ALIGN);
    }
    expect("q4 quantize w", tq_q4_quantize(nullptr, 300, &m, fake<uint8_t>(), fake<uint16_t>(), nullptr), TQ_ERR_NULL);
    expect("q4 quantize ldw", tq_q4_quantize(X, 299, &m, fake<uint8_t>(), fake<uint16_t>(), nullptr), TQ_ERR_SHAPE);
    expect("q4 quantize codes", tq_q4_quantize(X, 300, &m, nullptr, fake<uint16_t>(), nullptr), TQ_ERR_NULL);
    expect("q4 quantize matrix", tq_q4_quantize(X, 300, nullptr, fake<uint8_t>(), fake<uint16_t>(), nullptr), TQ_ERR_NULL);
    expect("q4 unpack w", tq_q4_unpack_fp16(&m, nullptr, nullptr), TQ_ERR_NULL);
    expect("q4 unpack matrix", tq_q4_unpack_fp16(nullptr, fake<uint16_t>(), nullptr), TQ_ERR_NULL);
  }

  // The cache's checks, through tq_kv_extend.
  {
    tq_kv_cache c = cache();
    expect("page bytes", (int)tq_kv_page_bytes(&c), 4 * 2 * 32 * (128 + 16));
    c.head_dim = 96; expect("head dim", extend(c), TQ_ERR_UNSUPPORTED);
    expect("page bytes of 96", (int)tq_kv_page_bytes(&c), 0);
    c = cache(); c.group = 256; expect("group", extend(c), TQ_ERR_UNSUPPORTED);
    c = cache(); c.head_dim = 64; c.group = 128; expect("group past D", extend(c), TQ_ERR_UNSUPPORTED);
    const int sizes[] = {0, -64, 16, 48, 2048};
    for (int ps : sizes) { c = cache(); c.page_size = ps; expect("page size", extend(c), TQ_ERR_UNSUPPORTED); }
    c = cache(); c.n_layers = 0; expect("layers", extend(c), TQ_ERR_UNSUPPORTED);
    c = cache(); c.n_kv_heads = 1025; expect("heads", extend(c), TQ_ERR_UNSUPPORTED);
    c = cache(); c.n_seqs = 0; expect("slots", extend(c), TQ_ERR_SHAPE);
    c = cache(); c.max_pages = 0; expect("max pages", extend(c), TQ_ERR_SHAPE);
    c = cache(); c.max_pages = TQ_KV_MAX_PAGES + 1; expect("max pages limit", extend(c), TQ_ERR_UNSUPPORTED);
    c = cache(); c.n_pages = 0; expect("pages", extend(c), TQ_ERR_SHAPE);
    c = cache(); c.n_pages = ((int64_t)1 << 30) + 1; expect("pages limit", extend(c), TQ_ERR_UNSUPPORTED);
    c = cache(); c.reserved = 1; expect("reserved", extend(c), TQ_ERR_SHAPE);
    c = cache(); c.data = nullptr; expect("data", extend(c), TQ_ERR_NULL);
    c = cache(); c.refs = nullptr; expect("refs", extend(c), TQ_ERR_NULL);
    c = cache(); c.data = fake<uint8_t>(8); expect("data align", extend(c), TQ_ERR_ALIGN);
    c = cache(); c.lens = fake<int32_t>(2); expect("lens align", extend(c), TQ_ERR_ALIGN);
    c = cache();
    expect("no cache", tq_kv_extend(nullptr, nullptr, nullptr, 1, fake<int32_t>(), nullptr, nullptr), TQ_ERR_NULL);
    expect("no rows", extend(c, 0), TQ_ERR_SHAPE);
    expect("rows past the slots", extend(c, 9), TQ_ERR_SHAPE);
    expect("rows past the limit", extend(c, TQ_KV_MAX_ROWS + 1, fake<const int32_t>()), TQ_ERR_SHAPE);
    expect("seqs align", extend(c, 8, fake<const int32_t>(2)), TQ_ERR_ALIGN);
    expect("starts", extend(c, 8, nullptr, nullptr), TQ_ERR_NULL);
    expect("free rows", tq_kv_free(&c, nullptr, 9, nullptr, nullptr), TQ_ERR_SHAPE);
    expect("free d_err align", tq_kv_free(&c, nullptr, 8, fake<int32_t>(1), nullptr), TQ_ERR_ALIGN);

    const size_t fork_ws = tq_kv_workspace_bytes(&c, 4), compact_ws = tq_kv_workspace_bytes(&c, 0);
    expect("fork workspace", fork_ws > 0, 1);
    expect("compact workspace", compact_ws >= 1200, 1);
    expect("workspace rows", (int)tq_kv_workspace_bytes(&c, -1), 0);
    const int32_t* I = fake<const int32_t>();
    expect("fork rows", tq_kv_fork(&c, I, I, 0, nullptr, fake<void>(), fork_ws, nullptr), TQ_ERR_SHAPE);
    expect("fork children", tq_kv_fork(&c, I, nullptr, 4, nullptr, fake<void>(), fork_ws, nullptr), TQ_ERR_NULL);
    expect("fork workspace size", tq_kv_fork(&c, I, I, 4, nullptr, fake<void>(), fork_ws - 1, nullptr), TQ_ERR_SHAPE);
    expect("fork workspace align", tq_kv_fork(&c, I, I, 4, nullptr, fake<void>(8), fork_ws, nullptr), TQ_ERR_ALIGN);
    expect("compact workspace null", tq_kv_compact(&c, nullptr, nullptr, compact_ws, nullptr), TQ_ERR_NULL);
    expect("compact workspace size", tq_kv_compact(&c, nullptr, fake<void>(), compact_ws - 1, nullptr), TQ_ERR_SHAPE);
    expect("copy rows", tq_kv_copy_pages(&c, I, I, 65536, nullptr, nullptr), TQ_ERR_SHAPE);
    expect("copy src", tq_kv_copy_pages(&c, nullptr, I, 4, nullptr, nullptr), TQ_ERR_NULL);

    const tq_kv_rows kv = {fake<const uint16_t>(), 512, 128}, none = {nullptr, 0, 0};
    auto append = [&](int layer, int rows, int tokens, int max_new, const int32_t* starts, const tq_kv_rows* k) {
      return (int)tq_kv_append(&c, layer, nullptr, starts, nullptr, rows, tokens, max_new, k, &kv, nullptr, nullptr);
    };
    expect("append layer", append(2, 8, 8, 1, I, &kv), TQ_ERR_SHAPE);
    expect("append rows", append(0, 9, 8, 1, I, &kv), TQ_ERR_SHAPE);
    expect("append tokens", append(0, 8, 0, 1, I, &kv), TQ_ERR_SHAPE);
    expect("append max_new", append(0, 8, 8, (1 << 26) + 1, I, &kv), TQ_ERR_SHAPE);
    expect("append starts", append(0, 8, 8, 1, nullptr, &kv), TQ_ERR_NULL);
    expect("append k", append(0, 8, 8, 1, I, nullptr), TQ_ERR_NULL);
    expect("append k data", append(0, 8, 8, 1, I, &none), TQ_ERR_NULL);
    expect("read out align", tq_kv_read(&c, 0, nullptr, I, nullptr, 8, 8, 1, fake<uint16_t>(8), fake<uint16_t>(), nullptr),
           TQ_ERR_ALIGN);
    expect("read out", tq_kv_read(&c, 0, nullptr, I, nullptr, 8, 8, 1, fake<uint16_t>(), nullptr, nullptr), TQ_ERR_NULL);
  }

  // Attention.
  {
    tq_kv_cache c = cache();
    tq_kv_attn a = attn();
    expect("attention null", tq_kv_attention(&c, 0, nullptr, nullptr), TQ_ERR_NULL);
    expect("attention layer", attend(c, a, 2), TQ_ERR_SHAPE);
    a = attn(); a.n_heads = 6; expect("heads of heads", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.n_rows = 9; expect("attention rows", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.max_q = 0; expect("max_q", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.max_len = -1; expect("max_len", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.window = -1; expect("window", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.n_heads = 4 * 16384; expect("query heads", attend(c, a), TQ_ERR_UNSUPPORTED);
    a = attn(); a.flags = 3; expect("attention flags", attend(c, a), TQ_ERR_UNSUPPORTED);
    a = attn(); a.scale = NAN; expect("scale", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.n_tokens = 1 << 28; expect("o past 2^31 rows", attend(c, a), TQ_ERR_UNSUPPORTED);
    a = attn(); a.q.data = nullptr; expect("q", attend(c, a), TQ_ERR_NULL);
    a = attn(); a.o = nullptr; expect("o", attend(c, a), TQ_ERR_NULL);
    a = attn(); a.o = fake<void>(8); expect("o align", attend(c, a), TQ_ERR_ALIGN);
    a = attn(); a.lse = fake<float>(2); expect("lse align", attend(c, a), TQ_ERR_ALIGN);
    c.max_pages = 1000;
    a = attn();
    const size_t need = tq_kv_attention_workspace_bytes(&c, &a);
    expect("workspace for a long cache", need > 0, 1);
    a.workspace = nullptr; expect("workspace", attend(c, a), TQ_ERR_NULL);
    a = attn(); a.workspace_bytes = need - 1; expect("workspace size", attend(c, a), TQ_ERR_SHAPE);
    a = attn(); a.workspace = fake<void>(8); expect("workspace align", attend(c, a), TQ_ERR_ALIGN);
    a = attn(); a.n_rows = 0; expect("workspace of bad arguments", (int)tq_kv_attention_workspace_bytes(&c, &a), 0);
    // more tiles than a launch takes
    c = cache();
    c.n_kv_heads = 1024;
    a = attn(); a.n_heads = 1024; a.n_rows = 1; a.n_tokens = 1 << 20; a.max_q = 1 << 20;
    a.n_tokens = 1 << 20;
    expect("tiles", attend(c, a), TQ_ERR_UNSUPPORTED);
  }

  std::printf("%s: %d failure(s)\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
