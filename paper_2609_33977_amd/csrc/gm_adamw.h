// One AdamW step on an fp32 parameter (decoupled decay, bias-corrected
// moments).  The coefficients are formed in fp64 on the host and rounded once
// (1 - beta directly, not from a rounded beta).
#pragma once

#include <hip/hip_runtime.h>

#include <math.h>

namespace gm {

struct AdamW {
  float lr, b1, omb1, b2, omb2, eps, decay, bc1, bc2;  // decay = 1 - lr weight_decay; bc = 1 / (1 - beta^t)
  __device__ __forceinline__ float step(float p, float g, float& m, float& v) const {
    m = b1 * m + omb1 * g;
    v = b2 * v + omb2 * g * g;
    return p * decay - lr * (m * bc1) / (sqrtf(v * bc2) + eps);
  }
};

inline AdamW make_adamw(double lr, double b1, double b2, double eps, double wd, int step) {
  AdamW o;
  o.lr = float(lr);
  o.b1 = float(b1);
  o.omb1 = float(1.0 - b1);
  o.b2 = float(b2);
  o.omb2 = float(1.0 - b2);
  o.eps = float(eps);
  o.decay = float(1.0 - lr * wd);
  o.bc1 = float(1.0 / (1.0 - pow(b1, double(step))));
  o.bc2 = float(1.0 / (1.0 - pow(b2, double(step))));
  return o;
}

}  // namespace gm
