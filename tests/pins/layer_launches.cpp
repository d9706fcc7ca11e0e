// Which kernels a call of the layers before the head launches, on the stand-in for the HIP runtime (fake_hip.h).  A line of standard input is a call, and
// is answered by a line: the kernels' names with their template arguments and grids, apart by " | ", or "refused" with its status.
//   linear out|grads  rows width outs  dtype act bits pad shift  arrays      (arrays: letters of what there is: b bias, g gate, r residual, p pre,
//                                                                             x d_x, w d_weight, d d_bias, e d_gate, a dropout)
//   rms norm|grads    rows width       dtype bits                arrays      (r residual, g d_gain, x d_x)
#define __hipRegisterFunction without_arguments
#include "fake_hip.h"
#undef __hipRegisterFunction
#include "ptchunk.h"

#include <iostream>
#include <sstream>

extern "C" void __hipRegisterFunction(void** mod, const void* host, char* a, const char* name, unsigned b, void* c, void* d, dim3* e, dim3* f, int* g) {
  without_arguments(mod, host, a, name, b, c, d, e, f, g);
  int st = 0;
  char* s = abi::__cxa_demangle(name, nullptr, nullptr, &st);
  std::string n = st == 0 && s ? s : name;
  free(s);
  for (const char* drop : {"(anonymous namespace)::", "pt_mfma::"})
    for (size_t at; (at = n.find(drop)) != std::string::npos;) n.erase(at, strlen(drop));
  const size_t k = n.find("k_"), end = n.find(">(");
  fake::kernels()[host] = n.substr(k, (end == std::string::npos ? n.find("(", k) : end + 1) - k);
}

// Addresses that nothing reads, each in a room of its own.
static uintptr_t room = 0;
static char* at(uint64_t shift) { return (char*)((room += uint64_t(1) << 40) + shift); }

static int linear(std::istream& in, bool grads) {
  pt_linear l = {};
  uint64_t pad, shift;
  int bits;
  std::string has;
  in >> l.rows >> l.width >> l.outs >> l.dtype >> l.act >> bits >> pad >> shift >> has;
  const auto there = [&](char c) { return has.find(c) != std::string::npos; };
  const uint64_t bytes = bits / 8;
  l.x = at(shift * bytes); l.weight = at(shift * bytes);
  l.x_stride = l.weight_stride = l.d_x_stride = l.d_weight_stride = l.width + pad;
  l.gate_stride = l.residual_stride = l.pre_stride = l.out_stride = l.d_out_stride = l.d_gate_stride = l.outs + pad;
  if (bits == 8) { l.x_scale = (float*)at(0); l.weight_scale = (float*)at(0); }
  if (there('b')) l.bias = at(0);
  if (there('g')) l.gate = at(2 * shift);
  if (there('r')) l.residual = at(2 * shift);
  if (there('p')) l.pre = at(2 * shift);
  if (there('a')) l.drop.p = 0.1;
  if (!grads) l.out = at(2 * shift);
  else {
    l.d_out = at(2 * shift);
    if (there('x')) l.d_x = at(2 * shift);
    if (there('w')) l.d_weight = at(2 * shift);
    if (there('d')) l.d_bias = at(0);
    if (there('e')) l.d_gate = at(2 * shift);
  }
  return (grads ? pt_linear_grads : pt_linear_out)(&l, at(0), ~uint64_t(0), nullptr);
}

static int rms(std::istream& in, bool grads) {
  pt_rms n = {};
  int bits;
  std::string has;
  in >> n.rows >> n.width >> n.dtype >> bits >> has;
  const auto there = [&](char c) { return has.find(c) != std::string::npos; };
  n.x = at(0); n.y = at(0); n.rstd = (float*)at(0); n.eps = 1e-5;
  n.x_stride = n.residual_stride = n.sum_stride = n.y_stride = n.d_y_stride = n.d_sum_stride = n.d_x_stride = n.width;
  if (bits == 8) n.y_scale = (float*)at(0);
  if (there('r')) { n.residual = at(0); n.sum = at(0); }
  if (!grads) return pt_rms_norm(&n, nullptr);
  n.d_y = at(0);
  if (there('x')) n.d_x = at(0);
  if (there('g')) n.d_gain = at(0);
  return pt_rms_grads(&n, at(0), ~uint64_t(0), nullptr);
}

int main() {
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string what, way;
    in >> what >> way;
    const size_t from = fake::ops.size();
    room = 0;
    const int rc = what == "linear" ? linear(in, way == "grads") : rms(in, way == "grads");
    if (rc != PT_OK) std::cout << "refused " << rc << " " << pt_last_error(nullptr);
    else
      for (size_t i = from; i < fake::ops.size(); ++i)
        if (fake::ops[i].what == "launch") std::cout << (i == from ? "" : " | ") << fake::ops[i].kernel << " grid " << fake::ops[i].grid.x;
    std::cout << std::endl;
  }
}
