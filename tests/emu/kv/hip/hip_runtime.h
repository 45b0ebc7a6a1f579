// TEST INFRASTRUCTURE ONLY.  What the kernels of the 4-bit key/value cache need beyond ../../hip/hip_runtime.h: the fp16 matrix
// instruction, a barrier of one wave, and a few small things.
#pragma once
#include "../../hip/hip_runtime.h"

struct float2 { float x, y; };
static inline float2 make_float2(float a, float b) { return float2{a, b}; }

namespace emu {
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
inline void wave_barrier() { g_ctx->wave_bar[t_threadIdx.x / 64]->arrive_and_wait(); }
extern h8 mfma_a[16][2][64], mfma_b[16][2][64];
// D[16 x 16] = A[16 x 32] B[32 x 16] + C: lane 16 g + n holds A[n][8 g + i], B[8 g + i][n] and C, D[4 g + r][n]
inline f4 mfma_16x16x32(h8 a, h8 b, f4 c)
{
    const unsigned tid = t_threadIdx.x, wave = tid / 64, lane = tid % 64, par = (t_opcount++) & 1u;
    mfma_a[wave][par][lane] = a;
    mfma_b[wave][par][lane] = b;
    wave_barrier();
    for (unsigned r = 0; r < 4; ++r) {
        float s = c[r];
        for (unsigned g = 0; g < 4; ++g)
            for (unsigned i = 0; i < 8; ++i)
                s += (float)mfma_a[wave][par][16 * g + 4 * (lane / 16) + r][i] * (float)mfma_b[wave][par][16 * g + lane % 16][i];
        c[r] = s;
    }
    return c;
}
}  // namespace emu
// shifts within rows of 16 lanes that bring in zeros; the other permutations are the common header's
static inline int emu_kv_dpp(uint32_t v, int ctrl)
{
    if (ctrl < 0x111 || ctrl > 0x11f) return (int)emu::exchange(v, -1, ctrl, 0);
    const unsigned lane = threadIdx.x % 64, by = (unsigned)ctrl & 15u, from = lane % 16 < by ? lane : lane - by;
    const uint32_t o = emu::exchange(v, (int)from, -1, 0);
    return lane % 16 < by ? 0 : (int)o;
}
#undef __builtin_amdgcn_update_dpp
#define __builtin_amdgcn_update_dpp(old, v, ctrl, rm, bm, bc) emu_kv_dpp((uint32_t)(v), (ctrl))
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) emu::mfma_16x16x32((a), (b), (c))
#define __builtin_amdgcn_wave_barrier() emu::wave_barrier()
#define __builtin_amdgcn_exp2f(x) exp2f(x)
static inline uint32_t atomicMax(uint32_t *p, uint32_t v)
{
    uint32_t o = __atomic_load_n(p, __ATOMIC_SEQ_CST);
    while (o < v && !__atomic_compare_exchange_n(p, &o, v, false, __ATOMIC_SEQ_CST, __ATOMIC_SEQ_CST)) {}
    return o;
}
