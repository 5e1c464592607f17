// Host-side state shared by the translation units of the library.
#pragma once

namespace gaf {

// Sets what gaf_last_launch_count() reports for the calling thread.
void set_last_launch_count(int launches);

// What gaf_test_set_wait_fault() left for the calling thread: attempts of a wait (0: the kernel's own limit), what is withheld.
unsigned int test_wait_limit();
int test_withhold();

}  // namespace gaf
