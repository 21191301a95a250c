// Arguments that the calls with polynomials and residuals check and scale alike (nonlinear.hip, epilogue.hip).
#pragma once
#include "api_args.h"
#include "step.h"

ckks_status check_poly(const ckks_poly *p, const char *what);
ckks_status check_scale(double s, const char *what, const char *name);
// n buffers of `polys` polynomials with at least `least` limbs and one positive scale
ckks_status check_list(const ckks_ctx *ctx, const ckks_buf *b, uint32_t n, uint32_t polys, uint32_t least,
                       const char *what, const char *name);
// the integer nearest to x, CKKS_ESCALE from 2^120
ckks_status scaled_int(double x, StepInt *out, const char *what, const char *name);
// t = (2 x - lo - hi) / (hi - lo) at scale s1: by = 2 / (hi - lo) s1, and the constant
ckks_status poly_map(const ckks_poly &p, double s1, double *by, StepInt *c, const char *what);
