// disco_dropout.hip -- dropout by a counter-based generator.
//
//   y = x factor where an entry's 16 bits are at least `out`, 0 elsewhere,
//   factor = 65536 / (65536 - out),
//
// the bits of entry c of row r being half c % 8 of Philox4x32-10 at the counter
// (c / 8, r, offset): the mask is a function of seed, offset and place, is never
// stored, and the gradient is the same call on dy.  Sixteen bits an entry instead
// of 32 halve the generator's work; the factor is that of the probability as it is
// taken, so the expectation stays exact.
//
// Each entry is read and written once, and the generator's ten rounds hide behind the
// loads: a thread takes one block of the generator, eight entries, as one load of 16 bytes
// (bf16) and leaves, and the card's other waves cover its wait.  32768 x 2048 bf16 (268 MB)
// take 48 us, 5.6 TB/s, where a copy of as many bytes moves 5.0 to 5.4 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "disco_blocks.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kThreads = 256;

struct Shape {
    Divisor chunks, tokens;  // of a row; rows of a batch item
    uint32_t all;            // chunks of all rows
};

template <typename T, bool EIGHTS>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutArgs a, Shape s) {
    const uint32_t i = group_index() * kThreads + threadIdx.x;
    if (i >= s.all) return;
    const uint32_t row = s.chunks.quotient(i), chunk = i - row * s.chunks.d;
    const uint32_t b = s.tokens.quotient(row), tok = row - b * s.tokens.d;
    const int64_t c = (int64_t)chunk * kChunk;
    const int left = (int)min((int64_t)kChunk, a.channels - c);
    const Raw<T> x = load_raw<T, EIGHTS>((const T*)a.x.p + b * a.x.sb + tok * a.x.st + c, left);
    const Words r = drop_words(a.drop, drop_offset(a.drop), row, chunk);
    float e[kChunk];
#pragma unroll
    for (int j = 0; j < kChunk; ++j) e[j] = stays(r, j, a.drop.out) ? x.at(j) * a.drop.factor : 0.0f;
    store_raw<T, EIGHTS>((T*)a.y.p + b * a.y.sb + tok * a.y.st + c, left, e);
}

template <typename T, bool EIGHTS>
hipError_t launch(const DropoutArgs& a, const Shape& s) {
    hipLaunchKernelGGL((k_dropout<T, EIGHTS>), grid_dim((s.all + kThreads - 1) / kThreads), dim3(kThreads), 0, a.stream, a, s);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a) {
    const int64_t chunks = (a.channels + kChunk - 1) / kChunk;
    Shape s;
    s.chunks = divisor((uint32_t)chunks);
    s.tokens = divisor((uint32_t)a.tokens);
    s.all = (uint32_t)(chunks * a.batch * a.tokens);
    const int tk = timing_begin("dropout", a.stream);
    const bool eights = a.channels % kChunk == 0;
    hipError_t err;
    if (a.bf16) err = eights ? launch<__bf16, true>(a, s) : launch<__bf16, false>(a, s);
    else err = eights ? launch<float, true>(a, s) : launch<float, false>(a, s);
    timing_end(tk, a.stream);
    return err;
}

}  // namespace disco
