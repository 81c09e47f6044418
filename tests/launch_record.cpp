// Records kernel launches instead of making them: loaded before the library, its hipLaunchKernel and
// __hipRegisterFunction stand in for the runtime's, so that launch shapes can be looked at without a GPU.
#include <cstdint>
#include <map>
#include <string>
#include <vector>

struct Dim3 {
  uint32_t x, y, z;
};
struct Launch {
  const char *name;
  Dim3 grid, block;
};

static std::map<const void *, std::string> &names() {
  static std::map<const void *, std::string> m;
  return m;
}
static std::vector<Launch> &launches() {
  static std::vector<Launch> v;
  return v;
}

extern "C" {

void __hipRegisterFunction(void **, const void *host, char *, const char *device, unsigned, void *, void *, void *, void *,
                           int *) {
  names()[host] = device;
}

int hipLaunchKernel(const void *f, Dim3 grid, Dim3 block, void **, size_t, void *) {
  const auto it = names().find(f);
  launches().push_back(Launch{it == names().end() ? "?" : it->second.c_str(), grid, block});
  return 0;
}

int recorded() { return (int)launches().size(); }
// name, and the six extents, of launch i
const char *recorded_launch(int i, uint32_t *extents) {
  const Launch &l = launches()[i];
  const uint32_t e[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
  for (int j = 0; j < 6; ++j) extents[j] = e[j];
  return l.name;
}
void forget() { launches().clear(); }
}
