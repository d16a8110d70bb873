// Frees plans on one thread while another one starts the library and shuts it down (without a GPU), as a program does whose garbage collector
// runs beside its last calls.  Built with AddressSanitizer by the test next to it: prints the answers that daris_free_plan gave.
#include <atomic>
#include <cstdio>
#include <thread>

#include "../../include/daris.h"
#include "../../include/daris_ops.h"

int main() {
  std::atomic<bool> over{false};
  long refused = 0, unknown = 0, other = 0;
  std::thread collector([&] {
    while (!over.load()) {
      const daris_status st = daris_free_plan(0);
      ++(st == DARIS_ESTATE ? refused : st == DARIS_ERANGE ? unknown : other);
    }
  });
  for (int i = 0; i < 20000; ++i)
    if (daris_init(0, 0, DARIS_VIRTUAL_TIME | DARIS_NO_DEVICE) != DARIS_OK || daris_shutdown() != DARIS_OK) return 3;
  over = true;
  collector.join();
  std::printf("%ld %ld %ld\n", refused, unknown, other);
  return 0;
}
