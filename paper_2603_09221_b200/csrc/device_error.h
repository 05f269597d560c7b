// Whether a bounded wait has given up, on the current device: one word for each source file whose kernels wait.
#pragma once

namespace ttc {

int attention_device_error(int* value);

} // namespace ttc
