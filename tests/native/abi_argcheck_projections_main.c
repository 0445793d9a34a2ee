/* Test driver (CPU only, no GPU needed): the rejection paths of svgear_linear, svgear_rotary and their backward passes, and
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

static void* const fake = (void*)0x10000;
static void* const odd = (void*)0x10001;
static void* const out = (void*)0x80000;
static void* const out2 = (void*)0x90000;
static const size_t big = (size_t)1 << 50;

static int lin(const void* x, const int64_t* xst, const void* w, int64_t ldw, svgear_dtype dt, int B, int64_t N, int k, int o,
               int act, const void* gate, const int64_t* gst, const void* res, const int64_t* rst, void* y, const int64_t* yst,
               size_t ws_bytes) {
  return svgear_linear(x, xst, w, ldw, NULL, dt, B, N, k, o, (svgear_act)act, gate, gst, res, rst, NULL, y, yst, fake, ws_bytes, NULL);
}

static void linear(void) {
  const int64_t s[2] = {1600, 16}, neg[2] = {1600, -16}, meet[2] = {1600, 15}, meet_b[2] = {1584, 16}, other[2] = {1600, 32};
  const int64_t inner_b[2] = {16, 32}, inner_meet[2] = {16, 31};
  const svgear_dtype H = SVGEAR_BF16;
  /* B = 2, N = 100, 16 to 16 */
  expect("linear: null x", lin(NULL, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: null strides", lin(fake, NULL, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: null w", lin(fake, s, NULL, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: null y", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, NULL, s, big), -1);
  expect("linear: null y strides", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, NULL, big), -1);
  expect("linear: B = 0", lin(fake, s, fake, 16, H, 0, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: N = 0", lin(fake, s, fake, 16, H, 2, 0, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: d_in = 0", lin(fake, s, fake, 16, H, 2, 100, 0, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: d_out < 0", lin(fake, s, fake, 16, H, 2, 100, 16, -3, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: d_in too large", lin(fake, s, fake, 1 << 22, H, 2, 100, (1 << 21) + 1, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: too many rows", lin(fake, s, fake, 16, H, 4, (int64_t)1 << 30, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: N past 32 bits", lin(fake, s, fake, 16, H, 1, (int64_t)1 << 40, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: w_stride < d_in", lin(fake, s, fake, 15, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: negative stride of x", lin(fake, neg, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  {
    const int64_t huge[2] = {INT64_MAX, INT64_MAX};
    expect("linear: strides of x that overflow", lin(fake, huge, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
    expect("linear: strides of y that overflow", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, huge, big), -1);
    expect("linear: w_stride that overflows", lin(fake, s, fake, INT64_MAX, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
    expect("linear_workspace: strides that overflow", (long long)svgear_linear_workspace(fake, huge, fake, 16, H, 2, 100, 16, 16), 0);
  }
  expect("linear: rows of y meet", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, meet, big), -1);
  expect("linear: batches of y meet", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, meet_b, big), -1);
  expect("linear: batches within tokens meet", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, inner_meet, big), -1);
  expect("linear: bad type", lin(fake, s, fake, 16, (svgear_dtype)2, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: bad activation", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 4, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: negative activation", lin(fake, s, fake, 16, H, 2, 100, 16, 16, -1, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: gate without strides", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, fake, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: residual without strides", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, fake, NULL, out, s, big), -1);
  expect("linear: negative stride of residual", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, fake, neg, out, s, big), -1);
  expect("linear: y over the residual with other strides", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, fake, other, fake, s, big), -1);
  expect("linear: y over x", lin(fake, s, (void*)0x20000, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, fake, s, big), -1);
  expect("linear: y over w", lin((void*)0x20000, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, fake, s, big), -1);
  expect("linear: pre over y",
         svgear_linear((void*)0x20000, s, (void*)0x30000, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, fake, fake, s, fake, big, NULL), -1);
  expect("linear_backward: dx over dy",
         svgear_linear_backward(fake, s, (void*)0x20000, s, (void*)0x30000, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, fake, s, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: dbias over dw",
         svgear_linear_backward(fake, s, (void*)0x20000, s, (void*)0x30000, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, (void*)0x40000, (void*)0x40000, NULL, fake, big, NULL), -1);
  expect("linear: x at an odd address", lin(odd, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, out, s, big), -1);
  expect("linear: y at an odd address", lin(fake, s, fake, 16, H, 2, 100, 16, 16, 0, NULL, NULL, NULL, NULL, odd, s, big), -1);
  {
    const int64_t packed[2] = {1700, 17};
    const size_t need = svgear_linear_workspace(fake, packed, fake, 17, H, 2, 100, 17, 16);
    expect("linear_workspace: unaligned rows need some", need > 0, 1);
    expect("linear: workspace too small", lin(fake, packed, fake, 17, H, 2, 100, 17, 16, 0, NULL, NULL, NULL, NULL, out, s, need - 1), -2);
    expect("linear: workspace null",
           svgear_linear(fake, packed, fake, 17, NULL, H, 2, 100, 17, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, NULL, out, s, NULL, big, NULL), -2);
    expect("linear: workspace not aligned",
           svgear_linear(fake, packed, fake, 17, NULL, H, 2, 100, 17, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, NULL, out, s, (void*)0x10010, big, NULL), -2);
  }
  expect("linear: bias at an odd address",
         svgear_linear(fake, s, fake, 16, odd, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, NULL, out, s, fake, big, NULL), -1);
  expect("linear: pre at an odd address",
         svgear_linear(fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, odd, out, s, fake, big, NULL), -1);
  expect("linear_workspace: aligned large calls need none", (long long)svgear_linear_workspace(fake, s, fake, 5120, H, 1, 75600, 5120, 15360), 0);
  expect("linear_workspace: invalid", (long long)svgear_linear_workspace(fake, s, fake, 16, H, 0, 100, 16, 16), 0);
  expect("linear_workspace: extreme returns", svgear_linear_workspace(fake, inner_b, odd, 1 << 21, SVGEAR_F32, 1 << 15, 1 << 15, 1 << 21, 1 << 21) > 0, 1);

  expect("linear_backward: nothing wanted",
         svgear_linear_backward(fake, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: null dy",
         svgear_linear_backward(NULL, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, out, s, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: dx without w",
         svgear_linear_backward(fake, s, fake, s, NULL, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, out, s, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: dx without strides",
         svgear_linear_backward(fake, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, out, NULL, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: dw without x",
         svgear_linear_backward(fake, s, NULL, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, out, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: activation without pre",
         svgear_linear_backward(fake, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_SILU, NULL, NULL, out, s, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: dgate without gate",
         svgear_linear_backward(fake, s, fake, s, fake, 16, fake, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, NULL, NULL, NULL, NULL, out, fake, big, NULL), -1);
  expect("linear_backward: dgate without pre",
         svgear_linear_backward(fake, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, fake, s, NULL, NULL, NULL, NULL, out, fake, big, NULL), -1);
  expect("linear_backward: rows of dx meet",
         svgear_linear_backward(fake, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, out, meet, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: w_stride < d_in",
         svgear_linear_backward(fake, s, fake, s, fake, 8, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, out, s, NULL, NULL, NULL, fake, big, NULL), -1);
  expect("linear_backward: workspace too small",
         svgear_linear_backward(fake, s, fake, s, fake, 16, NULL, H, 2, 100, 16, 16, SVGEAR_ACT_NONE, NULL, NULL, out, s, out2, (void*)0xa0000, NULL, fake, 16, NULL), -2);
  expect("linear_backward_workspace: extreme returns",
         svgear_linear_backward_workspace(fake, s, fake, s, fake, 1 << 21, SVGEAR_F32, 1 << 15, 1 << 15, 1 << 21, 1 << 21) > 0, 1);
  expect("linear_backward_workspace: invalid", (long long)svgear_linear_backward_workspace(fake, s, fake, s, fake, 16, H, 2, -1, 16, 16), 0);
}

typedef struct {
  int n, B, H, d;
  int64_t N, tail, first, pos_b;
  int sections[3];
  int64_t grid[3];
  const int64_t* gridp;
  const int32_t* pos;
  unsigned flags;
  float eps;
  svgear_dtype dt;
  const double* freq;
  int64_t st[2][3], dst[2][3];
  const void* src[2];
  void* out[2];
  const void* weight[2];
} Rot;

static Rot ordinary(void) {
  Rot r = {1, 2, 3, 64, 30, 6, 0, 0, {10, 11, 11}, {2, 3, 4}, NULL, NULL, SVGEAR_ROTARY_NORM_TOKEN, 1e-6f, SVGEAR_BF16, (const double*)0x10000,
           {{5760, 1920, 64}, {5760, 1920, 64}}, {{5760, 1920, 64}, {5760, 1920, 64}}, {(void*)0x10000, (void*)0x10000}, {(void*)0x20000, (void*)0x30000},
           {(void*)0x40000, (void*)0x40000}};
  return r;
}
static int rot(const Rot* r) {
  return svgear_rotary(r->n, r->src, r->st, r->out, r->dst, r->weight, r->dt, r->B, r->H, r->N, r->tail, r->d, r->freq, r->sections,
                       r->gridp ? r->gridp : r->grid, r->first, r->pos, r->pos_b, r->flags, r->eps, NULL);
}
static int back(const Rot* r, void* const* dweight, size_t ws_bytes) {
  return svgear_rotary_backward(r->n, r->src, r->st, r->src, r->st, r->out, r->dst, r->weight, dweight, r->dt, r->B, r->H, r->N, r->tail, r->d, r->freq,
                                r->sections, r->gridp ? r->gridp : r->grid, r->first, r->pos, r->pos_b, r->flags, r->eps, fake, ws_bytes, NULL);
}
#define REFUSED(what, change)        \
  do {                               \
    Rot r = ordinary();              \
    change;                          \
    expect("rotary: " what, rot(&r), -1); \
    expect("rotary_backward: " what, back(&r, NULL, big), -1); \
  } while (0)

static void rotary(void) {
  REFUSED("no tensors", r.n = 0);
  REFUSED("three tensors", r.n = 3);
  REFUSED("B = 0", r.B = 0);
  REFUSED("H = 129", r.H = 129);
  REFUSED("N = 0", r.N = 0);
  REFUSED("no rotated token", r.tail = 30);
  REFUSED("negative tail", r.tail = -1);
  REFUSED("d = 96", r.d = 96);
  REFUSED("bad type", r.dt = (svgear_dtype)5);
  REFUSED("too many tokens", (r.B = 1 << 16, r.N = 1 << 16));
  REFUSED("more pairs than half a head", r.sections[0] = 11);
  REFUSED("negative section", r.sections[1] = -1);
  REFUSED("sections that overflow", (r.sections[0] = 0x7fffffff, r.sections[1] = 0x7fffffff));
  REFUSED("no frequencies", r.freq = NULL);
  REFUSED("both norms", r.flags = 3u);
  REFUSED("unknown flag", r.flags = 8u);
  REFUSED("weight without a norm", r.flags = 0u);
  REFUSED("negative eps", r.eps = -1e-6f);
  REFUSED("NaN eps", r.eps = NAN);
  REFUSED("grid of no size", r.grid[1] = 0);
  REFUSED("grid past 32 bits", (r.grid[0] = 1 << 20, r.grid[1] = 1 << 20, r.grid[2] = 1 << 20));
  REFUSED("grid whose product overflows", (r.grid[0] = 0x7fffffff, r.grid[1] = 0x7fffffff, r.grid[2] = 0x7fffffff));
  REFUSED("tokens past the grid", r.first = 1);
  REFUSED("negative first", r.first = -1);
  REFUSED("first that overflows", r.first = INT64_MAX);
  REFUSED("positions at an odd address", r.pos = (const int32_t*)0x10002);
  REFUSED("positions of one batch entry in the next", (r.pos = (const int32_t*)0x10000, r.pos_b = 71));
  REFUSED("null tensor", r.src[0] = NULL);
  REFUSED("null output", r.out[0] = NULL);
  REFUSED("second tensor null", (r.n = 2, r.src[1] = NULL));
  REFUSED("input not 16-byte aligned", r.src[0] = (void*)0x10008);
  REFUSED("output not 16-byte aligned", r.out[0] = (void*)0x20008);
  REFUSED("weight not 16-byte aligned", r.weight[0] = (void*)0x40002);
  REFUSED("strides of no 16 bytes", r.st[0][2] = 65);
  REFUSED("negative stride", r.st[0][1] = -1920);
  REFUSED("a stride that overflows", r.st[0][0] = INT64_MAX - 7);
  REFUSED("an output's stride that overflows", r.dst[0][0] = INT64_MAX - 7);
  REFUSED("rows of the output meet", r.dst[0][2] = 56);
  REFUSED("heads of the output meet", r.dst[0][1] = 1856);
  REFUSED("two outputs at one address", (r.n = 2, r.out[1] = r.out[0]));
  REFUSED("an output over the other input", (r.n = 2, r.src[1] = (void*)0x50000, r.out[1] = (void*)0x30000, r.out[0] = (void*)0x50000));
  REFUSED("in place at other strides", (r.out[0] = (void*)r.src[0], r.dst[0][0] = 11520));
  REFUSED("batches of the output meet", r.dst[0][0] = 5696);
  {
    Rot r = ordinary();
    void* dw[2] = {fake, NULL};
    const size_t need = svgear_rotary_backward_workspace(1, 2, 3, 30, 64);
    expect("rotary_backward_workspace > 0", need > 0, 1);
    expect("rotary_backward: workspace too small", back(&r, dw, need - 1), -2);
    dw[0] = odd;
    expect("rotary_backward: dweight at an odd address", back(&r, dw, big), -1);
    dw[0] = fake;
    r.flags = 0;
    r.weight[0] = NULL;
    expect("rotary_backward: dweight without a norm", back(&r, dw, big), -1);
    expect("rotary_backward_workspace: extreme returns", svgear_rotary_backward_workspace(2, 1 << 10, 128, 1 << 20, 128) > 0, 1);
    expect("rotary_backward_workspace: invalid", (long long)svgear_rotary_backward_workspace(2, 1, 129, 10, 128), 0);
  }
}

int main(void) {
  linear();
  rotary();
  printf("%d wrong result(s)\n", failures);
  return failures;
}
