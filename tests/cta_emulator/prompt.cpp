// One CTA of the packed-prompt kernel in the emulator: key=value arguments, lens= the prompts' lengths, index:ms lists otherwise
#include "emu.h"
#include <sstream>
template <class T> T __shfl_sync(unsigned, T v, int from) { return emu::exchange(v, [from](T* a) { return a[from & 31]; }); }
#include "kernels.h"   // the kernels' sources as they are, without their includes

alignas(1024) uint8_t emu_smem[256 * 1024];
namespace kvc { uint8_t* smem_raw = emu_smem; }

static std::map<std::string, std::string> args;
static int num(const char* key, int other) { return args.count(key) ? atoi(args[key].c_str()) : other; }
static std::map<int, int> pairs(const char* key) {
  std::map<int, int> m;
  std::stringstream ss(args[key]);
  for (std::string item; std::getline(ss, item, ',');) m[atoi(item.c_str())] = atoi(item.c_str() + item.find(':') + 1);
  return m;
}

int main(int argc, char** argv) {
  for (int i = 1; i < argc; ++i) {
    const std::string a = argv[i];
    args[a.substr(0, a.find('='))] = a.substr(a.find('=') + 1);
  }
  emu::load_ms = pairs("load_ms");
  emu::suspend_ms = pairs("suspend_ms");
  emu::mma_us = num("mma_us", 20);
  emu::load_parts = 1;                                     // d = 64: one box per tile
  const int G = num("G", 1), Hkv = num("Hkv", 1), TOK = 128 / G;
  std::vector<kvc::PromptItem> items;
  std::stringstream ss(args["lens"]);
  int tokens = 0;
  for (std::string item; std::getline(ss, item, ',');) {
    const int n = atoi(item.c_str()), tiles = (n + TOK - 1) / TOK;
    for (int t = 0; t < tiles; t += 2)
      for (int h = 0; h < Hkv; ++h) items.push_back({tokens, n, t, h});
    tokens += n;
  }
  const int units = (int)items.size();
  items.back().head = ~items.back().head;
  items.push_back({1, 0, 0, 0});                           // where the units behind the first stand
  std::vector<int4> held(items.size());                    // (aligned as the kernel reads them)
  memcpy(held.data(), items.data(), items.size() * sizeof(int4));
  std::vector<char> ws(256);
  std::vector<__nv_bfloat16> out((size_t)tokens * G * Hkv * 64 + 16);
  std::vector<float> lse((size_t)tokens * G * Hkv, -1.f);   // (its rows tell which were written)
  kvc::PromptGeom g{G, G * Hkv, Hkv, units, 1.f, num("limit_ms", 20) * 1000000 / 1024, reinterpret_cast<kvc::PromptItem*>(held.data()), lse.data()};
  CUtensorMap tm;
  memset(&tm, 0, sizeof(tm));
  const int rc = emu::run(kvc::kAttnThreads, [&] { kvc::prompt_kernel<64>(tm, tm, tm, out.data(), ws.data(), g); });
  int unwritten = 0;
  for (float x : lse) unwritten += x == -1.f;
  printf("unwritten %d\nstatus %d\n", unwritten, *reinterpret_cast<int*>(ws.data()));
  return rc;
}
