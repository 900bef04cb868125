// Prints, for lines "ratio out_scale steps a b c a b c .." read from standard input, the bound that the scales of an orthogonalised update start
// from, and for every step what its products multiply with and the bound behind it.
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>

#include "../paper_2112_09335_b200/csrc/grouped_plan.hpp"

using namespace gcn_admm_grouped;

int main() {
  std::string line;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    std::string ratio;
    int steps;
    float out_scale;
    in >> ratio >> out_scale >> steps;
    double most = first_bound(std::stod(ratio));
    std::printf("%.17g", most);
    for (int i = 0; i < steps; ++i) {
      float a, b, c;
      in >> a >> b >> c;
      const Growth g = grow(most, a, b, c);
      const StepFactors f = step_factors(most, g, a, b, c, i + 1 == steps, out_scale);
      most = bound_behind(g);
      std::printf(" %.9g %.9g %.9g %.9g %.9g %.9g %.17g", f.gram, f.square, f.linear, f.diagonal, f.move, f.scale, most);
    }
    std::printf("\n");
  }
}
