// ee_paged_attn_f32.hip -- attention of new rows over the paged cache, fp32.
#include "ee_paged_attn.h"

// One wave per (row, query head): 64 positions at a time, a lane each for the scores, then the lanes share out the features.
template <class T>
__global__ void __launch_bounds__(256)
k_paged_attn(PagedView pv, StepView st, HeadsView q, HeadsView out, int Hq, float scale, int window) {
    __shared__ float qs[4][256];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, hd = pv.hd, ps = pv.page_size;
    const int64_t id = (int64_t)blockIdx.x * 4 + w;
    const int t = (int)(id / Hq), h = (int)(id % Hq);
    if (t >= st.n_tokens) return;
    const int s = seq_of_slot(st, t, 1, 0);
    const SeqRows sr = seq_rows(st, s);
    if (t < sr.row0 || t >= sr.row0 + sr.n) return;
    const int p = sr.len - sr.n + t - sr.row0;
    const T* qr = (const T*)q.p + t * q.ts + h * q.hs;
    for (int i = lane; i < hd; i += 64) qs[w][i] = to_f32(qr[i]) * scale;
    __builtin_amdgcn_wave_barrier();
    const int lo = window > 0 ? max(0, p - window + 1) : 0, g = h / (Hq / pv.n_kv_heads);
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    bool seen = false;
    for (int c = lo; c <= p; c += 64) {
        const int j = c + lane;
        const T* blk = nullptr;
        if (j <= p) {
            const int page = st.pages[(int64_t)s * st.pages_per_seq + j / ps];
            if (page >= 0 && page < pv.n_pages) blk = (const T*)pv.pool + ((int64_t)page * pv.n_kv_heads + g) * (2LL * ps * hd);
            else if (st.status) atomicOr(st.status, 1);
        }
        float x = -INFINITY;
        if (blk) {
            x = 0.f;
            for (int i = 0; i < hd; ++i) x = fmaf(qs[w][i], to_f32(blk[page_k<T>(j % ps, i, hd, ps)]), x);
        }
        seen = seen || __any(blk != nullptr);
        float mx = x;
        for (int d = 32; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 64));
        mx = fmaxf(mx, m);
        const float ref = mx == -INFINITY ? 0.f : mx, a = expf(m - ref);
        const float e = blk ? expf(x - ref) : 0.f;
        float sum = e;
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
        l = l * a + sum;
        m = mx;
        for (int k = 0; k < 4; ++k) o[k] *= a;
        for (int jj = 0; jj < 64; ++jj) {
            const uint64_t b = (uint64_t)blk;
            const uint64_t at = ((uint64_t)(uint32_t)__shfl((int)(b >> 32), jj, 64) << 32) | (uint32_t)__shfl((int)b, jj, 64);
            if (at == 0) continue;
            const float ej = __shfl(e, jj, 64);
            for (int k = 0; k < 4; ++k)
                if (lane + 64 * k < hd) o[k] = fmaf(ej, to_f32(((const T*)at)[page_v<T>((c + jj) % ps, lane + 64 * k, hd, ps)]), o[k]);
        }
    }
    T* dst = (T*)out.p + t * out.ts + h * out.hs;
    for (int k = 0; k < 4; ++k)
        if (lane + 64 * k < hd) dst[lane + 64 * k] = from_f32<T>(seen ? o[k] / l : 0.f);
}

int f32_paged_attention(const PagedView& pv, const StepView& st, const HeadsView& q, const HeadsView& out, int n_q_heads, float scale,
                        int window, hipStream_t s) {
    const int64_t waves = (int64_t)st.n_tokens * n_q_heads;
    hipLaunchKernelGGL(k_paged_attn<float>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, pv, st, q, out, n_q_heads, scale, window);
    EE_LAUNCH_CHECK();
    return EE_OK;
}
