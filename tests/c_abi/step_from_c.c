/* A training step's end driven from plain C: norm, clipping and AdamW over three tensors through the C ABI, compared with the
 * same formulas in double on the host. */
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <cuda_runtime_api.h>

#include "director.h"

#define N_TENSORS 3
static const int64_t kLength[N_TENSORS] = {5000, 0, 777};

static void* to_device(const void* src, size_t bytes) {
    void* p = NULL;
    if (cudaMalloc(&p, bytes ? bytes : 16) != cudaSuccess) exit(2);
    if (bytes && cudaMemcpy(p, src, bytes, cudaMemcpyHostToDevice) != cudaSuccess) exit(2);
    return p;
}
static int off(double got, double want, double rel) { return !(fabs(got - want) <= rel * fabs(want) + 1e-12); }

int main(void) {
    director_tensor grads[N_TENSORS], out[N_TENSORS];
    director_param params[N_TENSORS];
    float *g[N_TENSORS], *w[N_TENSORS], *back = malloc(5000 * sizeof(float));
    double square = 0.0;
    memset(grads, 0, sizeof grads);
    memset(out, 0, sizeof out);
    memset(params, 0, sizeof params);
    for (int i = 0; i < N_TENSORS; ++i) {
        const int64_t n = kLength[i];
        g[i] = malloc((size_t)(n + 1) * sizeof(float));
        w[i] = malloc((size_t)(n + 1) * sizeof(float));
        for (int64_t j = 0; j < n; ++j) {
            g[i][j] = (float)((j * 37 + i) % 101 - 50) * 0.01f;
            w[i][j] = (float)((j * 53 + i) % 89 - 44) * 0.02f;
            square += (double)g[i][j] * g[i][j];
        }
        grads[i].data = to_device(g[i], (size_t)n * 4);
        out[i].data = to_device(NULL, 0);
        if (n) {
            cudaFree(out[i].data);
            out[i].data = to_device(g[i], (size_t)n * 4);
            cudaMemset(out[i].data, 0xFF, (size_t)n * 4);
        }
        grads[i].numel = out[i].numel = params[i].numel = n;
        grads[i].type = out[i].type = params[i].type = DIRECTOR_FP32;
        params[i].weight = to_device(w[i], (size_t)n * 4);
        memset(back, 0, 5000 * sizeof(float));
        params[i].exp_avg = to_device(back, (size_t)n * 4);
        params[i].exp_avg_sq = to_device(back, (size_t)n * 4);
    }
    const double norm = sqrt(square), max_norm = 0.25 * norm;
    int64_t zero = 0, done = 0;
    int32_t none = 0, status = -1;
    float got = 0.0f;
    float* d_norm = to_device(&got, 4);
    int64_t* d_steps = to_device(&zero, 8);
    int32_t* d_status = to_device(&none, 4);
    void* work = to_device(NULL, 0);
    cudaFree(work);
    if (cudaMalloc(&work, (size_t)director_grad_workspace_bytes()) != cudaSuccess) return 2;
    int bad = 0;

    bad += director_grad_norm(N_TENSORS, grads, d_norm, NULL, NULL) != DIRECTOR_OK;       /* small: no workspace */
    cudaMemcpy(&got, d_norm, 4, cudaMemcpyDeviceToHost);
    bad += off(got, norm, 1e-6);

    bad += director_clip_grads(N_TENSORS, grads, out, (float)max_norm, d_norm, work, NULL) != DIRECTOR_OK;
    for (int i = 0; i < N_TENSORS; ++i) {
        cudaMemcpy(back, out[i].data, (size_t)kLength[i] * 4, cudaMemcpyDeviceToHost);
        for (int64_t j = 0; j < kLength[i]; ++j) bad += off(back[j], 0.25 * g[i][j], 1e-5);
    }

    director_adamw h = {1e-2, 0.9, 0.99, 1e-8, 0.1, max_norm};
    bad += director_adamw_step(N_TENSORS, grads, params, &h, NULL, d_steps, d_norm, d_status, work, NULL) != DIRECTOR_OK;
    for (int i = 0; i < N_TENSORS; ++i) {
        cudaMemcpy(back, params[i].weight, (size_t)kLength[i] * 4, cudaMemcpyDeviceToHost);
        for (int64_t j = 0; j < kLength[i]; ++j) {           /* the first step: m / (1 - beta1) = g', v / (1 - beta2) = g'^2 */
            const double x = 0.25 * g[i][j], want = w[i][j] - 1e-3 * w[i][j] - 1e-2 * x / (fabs(x) + 1e-8);
            bad += fabs(back[j] - want) > 1e-6;
        }
    }
    cudaMemcpy(&done, d_steps, 8, cudaMemcpyDeviceToHost);
    cudaMemcpy(&status, d_status, 4, cudaMemcpyDeviceToHost);
    bad += done != 1 || status != 0;
    h.beta1 = 1.0;
    bad += director_adamw_step(N_TENSORS, grads, params, &h, NULL, d_steps, d_norm, d_status, work, NULL) != DIRECTOR_ERR_INVALID_ARG;
    printf("%d mismatches\n", bad);
    return bad != 0;
}
