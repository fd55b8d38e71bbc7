// Cosine and sine of x, |x| <= pi / 4, by their series: the first term left out is below 2^-24 (32 bits) or 2^-54 (64 bits) of the result.
// The same code on the host, where the bounds are checked in more bits.
#pragma once

#ifdef __HIPCC__
#define AA_TURN __host__ __device__ __forceinline__
#else
#define AA_TURN inline
#endif

namespace aa {

template <class S> AA_TURN void series32(S x, S* c, S* s) {
    const S y = x * x;
    *c = 1 + y * (S(-1) / 2 + y * (S(1) / 24 + y * (S(-1) / 720 + y * (S(1) / 40320 + y * (S(-1) / 3628800)))));
    *s = x + x * y * (S(-1) / 6 + y * (S(1) / 120 + y * (S(-1) / 5040 + y * (S(1) / 362880))));
}
template <class S> AA_TURN void series64(S x, S* c, S* s) {
    const S y = x * x;
    *c = 1 + y * (S(-1) / 2 + y * (S(1) / 24 + y * (S(-1) / 720 + y * (S(1) / 40320 + y * (S(-1) / 3628800 +
             y * (S(1) / 479001600 + y * (S(-1) / 87178291200ll + y * (S(1) / 20922789888000ll))))))));
    *s = x + x * y * (S(-1) / 6 + y * (S(1) / 120 + y * (S(-1) / 5040 + y * (S(1) / 362880 + y * (S(-1) / 39916800 +
             y * (S(1) / 6227020800ll + y * (S(-1) / 1307674368000ll + y * (S(1) / 355687428096000ll))))))));
}

AA_TURN void series(float x, float* c, float* s) { series32(x, c, s); }
AA_TURN void series(double x, double* c, double* s) { series64(x, c, s); }

}  // namespace aa
