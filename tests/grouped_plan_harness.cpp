// Prints what the host side of the grouped products and orthogonalised updates says about calls read from standard input, one a line:
//   p type out_type groups rows k n transposed ldx ldw stride_w ldy        -> "ok ldx ldw stride_w ldy" or what is wrong
//   t type out_type groups rows ka nb ldx ldy lddw stride_dw               -> "ok ldx ldy lddw stride_dw" or what is wrong
//   o type out_type batch rows cols steps eps scale a b c                  -> "ok" or what is wrong (the same coefficients every step)
//   g most a b c                                                           -> largest value and factor of a step
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "../paper_2112_09335_b200/csrc/grouped_plan.hpp"

using namespace gcn_admm_grouped;

int main() {
  std::string line;
  alignas(16) static char somewhere[64];
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    char what;
    in >> what;
    if (what == 'p') {
      Product p{};
      p.x = p.w = p.y = somewhere;
      in >> p.type >> p.out_type >> p.groups >> p.rows >> p.k >> p.n >> p.transposed >> p.ldx >> p.ldw >> p.stride_w >> p.ldy;
      int shift = 0;
      if (in >> shift) p.x = somewhere + shift;
      const char* wrong = check(p);
      if (wrong) std::printf("%s\n", wrong);
      else std::printf("ok %lld %lld %lld %lld\n", p.ldx, p.ldw, p.stride_w, p.ldy);
    } else if (what == 't') {
      ProductTn p{};
      p.x = p.y = p.dw = somewhere;
      in >> p.type >> p.out_type >> p.groups >> p.rows >> p.ka >> p.nb >> p.ldx >> p.ldy >> p.lddw >> p.stride_dw;
      const char* wrong = check(p);
      if (wrong) std::printf("%s\n", wrong);
      else std::printf("ok %lld %lld %lld %lld\n", p.ldx, p.ldy, p.lddw, p.stride_dw);
    } else if (what == 'o') {
      Orthogonal p{};
      p.g = p.out = somewhere;
      float c[3];
      std::string eps, scale;
      in >> p.type >> p.out_type >> p.batch >> p.rows >> p.cols >> p.steps >> eps >> scale >> c[0] >> c[1] >> c[2];
      p.eps = std::stof(eps);
      p.scale = std::stof(scale);
      std::vector<float> all;
      for (int i = 0; i < p.steps; ++i) all.insert(all.end(), c, c + 3);
      p.coefficients = all.data();
      const char* wrong = check(p);
      std::printf("%s\n", wrong ? wrong : "ok");
    } else if (what == 'g') {
      double most, a, b, c;
      in >> most >> a >> b >> c;
      const Growth g = grow(most, a, b, c);
      std::printf("%.17g %.17g\n", g.value, g.factor);
    }
  }
}
