/* Test driver (CPU only, no GPU needed): the rejection paths of svgear_layer_norm, svgear_attention and their backward passes, and
 * their workspace queries at ordinary and extreme sizes, against a copy of the library whose host code runs under sanitizers.
 * Device pointers are fakes that a correct argument check never dereferences. Prints one line per check and returns the number
 * of wrong results. */
#include <math.h>
#include <stdio.h>

#include "svgear.h"

static int failures = 0;
static void expect(const char* what, long long got, long long want) {
  printf("%-78s %lld%s\n", what, got, got == want ? "" : "   <-- WRONG");
  if (got != want) ++failures;
}

static char* const fake = (char*)0x10000;
static void* const odd = (void*)0x10001;
static char* const out = (char*)0x80000;
static const svgear_dtype BF = SVGEAR_BF16;

/* ---- layer norm: 2 x 100 tokens of 16 */
typedef struct {
  const void *x, *w, *b, *scale, *shift;
  const int64_t *xst, *sst, *hst, *yst;
  int dt, B;
  int64_t N;
  int c;
  float eps;
  void* y;
} norm_args;
static const int64_t rows[2] = {1600, 16}, none[2] = {16, 0}, neg[2] = {1600, -16}, meet[2] = {1600, 15}, huge[2] = {INT64_MAX, INT64_MAX};
static norm_args norm(void) {
  norm_args a = {fake, NULL, NULL, NULL, NULL, rows, none, none, rows, SVGEAR_BF16, 2, 100, 16, 1e-6f, out};
  return a;
}
static int call(norm_args a) {
  return svgear_layer_norm(a.x, a.xst, a.w, a.b, a.scale, a.sst, a.shift, a.hst, (svgear_dtype)a.dt, a.B, a.N, a.c, a.eps, a.y, a.yst, NULL);
}
#define REFUSED(what, change)          \
  do {                                 \
    norm_args a = norm();              \
    change;                            \
    expect("norm: " what, call(a), -1); \
  } while (0)

static void layer_norm(void) {
  REFUSED("null x", a.x = NULL);
  REFUSED("null strides", a.xst = NULL);
  REFUSED("null y", a.y = NULL);
  REFUSED("null y strides", a.yst = NULL);
  REFUSED("unaligned x", a.x = odd);
  REFUSED("unaligned weight", a.w = odd);
  REFUSED("unaligned shift", a.shift = odd);
  REFUSED("negative stride", a.xst = neg);
  REFUSED("strides that overflow", a.xst = huge);
  REFUSED("rows of y meet", a.yst = meet);
  REFUSED("all rows of y one", a.yst = none);
  REFUSED("B = 0", a.B = 0);
  REFUSED("N = 0", a.N = 0);
  REFUSED("too many tokens", a.N = (int64_t)1 << 30);
  REFUSED("N past 32 bits", a.N = (int64_t)1 << 40);
  REFUSED("c = 0", a.c = 0);
  REFUSED("c < 0", a.c = -8);
  REFUSED("c too large", a.c = (1 << 15) + 1);
  REFUSED("bad type", a.dt = 2);
  REFUSED("a type far out of range", a.dt = 0x7fffffff);
  REFUSED("negative eps", a.eps = -1.f);
  REFUSED("NaN eps", a.eps = NAN);
  REFUSED("infinite eps", a.eps = INFINITY);
  REFUSED("scale without strides", (a.scale = fake + 64, a.sst = NULL));
  REFUSED("y over the weight", a.w = out);
  REFUSED("y over the shift", a.shift = out);
  REFUSED("y over x at other strides", (a.x = out, a.xst = none));
}

static int norm_back(int modulation, const void* scale, const int64_t* sst, void* dx, const int64_t* dxst, void* dw, void* ds, size_t bytes) {
  return svgear_layer_norm_backward(fake, rows, fake + 4096, rows, NULL, NULL, scale, sst, modulation, BF, 2, 100, 16, 1e-6f, dx, dxst, dw, NULL, ds,
                                    NULL, fake + 65536, bytes, NULL);
}
static void layer_norm_backward(void) {
  const size_t big = (size_t)1 << 40;
  expect("norm_backward: nothing wanted", norm_back(0, NULL, NULL, NULL, NULL, NULL, NULL, big), -1);
  expect("norm_backward: an unknown modulation", norm_back(3, NULL, NULL, out, rows, NULL, NULL, big), -1);
  expect("norm_backward: a negative modulation", norm_back(-1, NULL, NULL, out, rows, NULL, NULL, big), -1);
  expect("norm_backward: scale without modulation", norm_back(0, fake + 64, none, out, rows, NULL, NULL, big), -1);
  expect("norm_backward: dscale without modulation", norm_back(0, NULL, NULL, out, rows, NULL, out + 64, big), -1);
  expect("norm_backward: a token's scale as an entry's", norm_back(1, fake + 64, rows, out, rows, NULL, NULL, big), -1);
  expect("norm_backward: dx without strides", norm_back(0, NULL, NULL, out, NULL, NULL, NULL, big), -1);
  expect("norm_backward: rows of dx meet", norm_back(0, NULL, NULL, out, meet, NULL, NULL, big), -1);
  expect("norm_backward: dx over x", norm_back(0, NULL, NULL, fake + 4096, rows, NULL, NULL, big), -1);
  expect("norm_backward: dx over dy at other strides", norm_back(0, NULL, NULL, fake, (const int64_t[2]){3200, 32}, NULL, NULL, big), -1);
  expect("norm_backward: dweight over dx", norm_back(0, NULL, NULL, out, rows, out, NULL, big), -1);
  expect("norm_backward: dweight unaligned", norm_back(0, NULL, NULL, out, rows, odd, NULL, big), -1);
  expect("norm_backward: no room for the sums", norm_back(0, NULL, NULL, out, rows, out + 64, NULL, 8), -2);
  expect("norm_backward_workspace: invalid", (long long)svgear_layer_norm_backward_workspace(BF, 2, 100, 0, 0), 0);
  expect("norm_backward_workspace: an unknown modulation", (long long)svgear_layer_norm_backward_workspace(BF, 2, 100, 16, 7), 0);
  {
    const size_t w = svgear_layer_norm_backward_workspace(BF, 1, 75600, 5120, SVGEAR_NORM_BATCH);
    expect("norm_backward_workspace: two sums of a row at least, a GB at most", w >= 2 * 5120 * 4 && w < ((size_t)1 << 30), 1);
  }
}

/* ---- attention: 2 x 4 heads (2 of keys), 100 queries, 50 keys of 64 */
typedef struct {
  const void *q, *k, *v;
  const int64_t *qst, *kst, *vst, *ost;
  int dt, B, H, Hk;
  int64_t Nq, Nk;
  int d;
  float scale, cap;
  unsigned flags;
  int n_docs;
  const int32_t *qo, *ko, *prefix;
  void* o;
  float* lse;
  size_t bytes;
} att_args;
static const int64_t q3[3] = {25600, 6400, 64}, k3[3] = {6400, 3200, 64}, n3[3] = {25600, -6400, 64}, o3[3] = {25600, 6400, 65}, m3[3] = {25600, 6400, 56},
                     far3[3] = {6400, 3200, (1 << 24) + 8}, h3[3] = {INT64_MAX, INT64_MAX, INT64_MAX};
static att_args att(void) {
  att_args a = {fake, fake + 4096, fake + 8192, q3, k3, k3, q3, SVGEAR_BF16, 2, 4, 2, 100, 50, 64, 0.125f, 0.f, 0, 0, NULL, NULL, NULL, out, NULL, (size_t)1 << 40};
  return a;
}
static int call_att(att_args a) {
  return svgear_attention(a.q, a.qst, a.k, a.kst, a.v, a.vst, (svgear_dtype)a.dt, a.B, a.H, a.Hk, a.Nq, a.Nk, a.d, a.scale, a.cap, NULL, a.flags,
                          a.n_docs, a.qo, a.ko, a.prefix, a.o, a.ost, a.lse, fake + 65536, a.bytes, NULL);
}
#define NOT(what, change)                       \
  do {                                          \
    att_args a = att();                         \
    change;                                     \
    expect("attention: " what, call_att(a), -1); \
  } while (0)

static void attention(void) {
  const int32_t* off = (const int32_t*)(fake + 32768);
  NOT("null q", a.q = NULL);
  NOT("null k", a.k = NULL);
  NOT("null v", a.v = NULL);
  NOT("null o", a.o = NULL);
  NOT("null strides of q", a.qst = NULL);
  NOT("null strides of o", a.ost = NULL);
  NOT("q not on 16 bytes", a.q = fake + 8);
  NOT("v not on 16 bytes", a.v = fake + 2);
  NOT("o not on 16 bytes", a.o = out + 4);
  NOT("lse not on 4 bytes", a.lse = (float*)odd);
  NOT("a negative stride", a.qst = n3);
  NOT("a stride of no whole 16 bytes", a.kst = o3);
  NOT("strides that overflow", a.vst = h3);
  NOT("keys too far apart", a.kst = far3);
  NOT("rows of o meet", a.ost = m3);
  NOT("bad type", a.dt = 2);
  NOT("B = 0", a.B = 0);
  NOT("H = 0", a.H = 0);
  NOT("Hk = 0", a.Hk = 0);
  NOT("Hk that does not divide H", a.Hk = 3);
  NOT("more heads of keys than of queries", a.Hk = 8);
  NOT("no queries", a.Nq = 0);
  NOT("no keys", a.Nk = 0);
  NOT("too many queries", a.Nq = ((int64_t)1 << 30) + 1);
  NOT("Nk past 32 bits", a.Nk = (int64_t)1 << 40);
  NOT("too many rows of a head", (a.Nq = (int64_t)1 << 30));
  NOT("d = 32", a.d = 32);
  NOT("d = 0", a.d = 0);
  NOT("NaN scale", a.scale = NAN);
  NOT("infinite scale", a.scale = INFINITY);
  NOT("negative cap", a.cap = -1.f);
  NOT("infinite cap", a.cap = INFINITY);
  NOT("NaN cap", a.cap = NAN);
  NOT("an unknown flag", a.flags = 4);
  NOT("a prefix without causal", a.prefix = off);
  NOT("documents without offsets", a.n_docs = 2);
  NOT("offsets without documents", (a.qo = off, a.ko = off));
  NOT("several documents of the keys alone", (a.n_docs = 2, a.ko = off));
  NOT("a negative number of documents", (a.n_docs = -1, a.qo = off, a.ko = off));
  NOT("too many documents", (a.n_docs = (1 << 20) + 1, a.qo = off, a.ko = off));
  NOT("offsets not on 4 bytes", (a.n_docs = 1, a.ko = (const int32_t*)odd));
  NOT("o over q", a.o = fake);
  NOT("o over v", a.o = fake + 8192);
  NOT("lse over o", a.lse = (float*)out);
  NOT("lse over k", a.lse = (float*)(fake + 4096));
  {
    att_args a = att();
    a.bytes = 8;
    a.Nk = 5000;
    expect("attention: no room for the parts", call_att(a), -2);
  }
  expect("attention_workspace: invalid", (long long)svgear_attention_workspace(BF, 2, 4, 3, 100, 50, 64, 0), 0);
  expect("attention_workspace: none for a query and few keys", (long long)svgear_attention_workspace(BF, 2, 4, 2, 1, 60, 64, 0), 0);
  {
    const size_t w = svgear_attention_workspace(BF, 1, 40, 40, 75600, 512, 128, 1);
    expect("attention_workspace: no parts for many queries", w >= (size_t)40 * 591 * 16 && w <= (size_t)40 * 600 * 16, 1);
  }
  {
    const size_t w = svgear_attention_workspace(BF, 8, 40, 8, 1, 32760, 128, 1);
    expect("attention_workspace: parts of single tokens", w >= (size_t)2 * 320 * 520 && w <= (size_t)64 * 320 * 520 + 512, 1);
    expect("attention_workspace: sizes at their limits", svgear_attention_workspace(SVGEAR_F32, 1, 1, 1, (int64_t)1 << 30, (int64_t)1 << 30, 128, 0),
           (long long)1 << 29);
  }
}

static int att_back(const int64_t* ost, const float* lse, void* dq, void* dk, void* dv, const int64_t* dst, size_t bytes) {
  return svgear_attention_backward(fake + 256, q3, fake, q3, fake + 4096, k3, fake + 8192, k3, fake + 16384, ost, lse, BF, 2, 4, 2, 100, 50, 64, 0.125f,
                                   0.f, NULL, 0, 0, NULL, NULL, NULL, dq, dq ? q3 : NULL, dk, dst, dv, dst, fake + 65536, bytes, NULL);
}
static void attention_backward(void) {
  const size_t big = (size_t)1 << 40;
  const float* lse = (const float*)(fake + 20480);
  expect("attention_backward: nothing wanted", att_back(q3, lse, NULL, NULL, NULL, NULL, big), -1);
  expect("attention_backward: dk without dv", att_back(q3, lse, out, out + 4096, NULL, k3, big), -1);
  expect("attention_backward: dv without dk", att_back(q3, lse, out, NULL, out + 4096, k3, big), -1);
  expect("attention_backward: dk without strides", att_back(q3, lse, out, out + 4096, out + 8192, NULL, big), -1);
  expect("attention_backward: no lse", att_back(q3, NULL, out, out + 4096, out + 8192, k3, big), -1);
  expect("attention_backward: o without strides", att_back(NULL, lse, out, out + 4096, out + 8192, k3, big), -1);
  expect("attention_backward: dq over q", att_back(q3, lse, fake, out + 4096, out + 8192, k3, big), -1);
  expect("attention_backward: dk over dv", att_back(q3, lse, out, out + 4096, out + 4096, k3, big), -1);
  expect("attention_backward: dv over o", att_back(q3, lse, out, out + 4096, fake + 16384, k3, big), -1);
  expect("attention_backward: rows of dk meet", att_back(q3, lse, out, out + 4096, out + 8192, m3, big), -1);
  expect("attention_backward: no room", att_back(q3, lse, out, out + 4096, out + 8192, k3, 64), -2);
  expect("attention_backward_workspace: invalid", (long long)svgear_attention_backward_workspace(BF, 2, 4, 2, 0, 50, 64, 0), 0);
  expect("attention_backward_workspace: a number for each query at least",
         svgear_attention_backward_workspace(BF, 1, 16, 16, 9450, 9450, 128, 4) >= (size_t)16 * 9450 * 4, 1);
}

int main(void) {
  layer_norm();
  layer_norm_backward();
  attention();
  attention_backward();
  printf("%d wrong result(s)\n", failures);
  return failures;
}
