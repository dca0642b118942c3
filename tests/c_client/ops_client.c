/* A plain C program on the handle-free operators of include/zoa.h: argv[1] holds m, n, k (int64), x [m, k] and
 * w [n, k] (binary32); argv[2] receives Q(x) Q(w)^T [m, n] (binary32), and the loss and gradient of the result's rows
 * against the single listed token 0. */
#include <cuda_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "zoa.h"

#define CHECK(call)                                                              \
    do {                                                                         \
        const int status_ = (int)(call);                                         \
        if (status_ != 0) {                                                      \
            fprintf(stderr, "%s: %d (%s)\n", #call, status_, zoa_ops_last_error()); \
            return 1;                                                            \
        }                                                                        \
    } while (0)

static float *on_device(const float *host, size_t count)
{
    void *p = NULL;
    if (cudaMalloc(&p, count * sizeof(float)) != cudaSuccess) return NULL;
    if (host && cudaMemcpy(p, host, count * sizeof(float), cudaMemcpyHostToDevice) != cudaSuccess) return NULL;
    return (float *)p;
}

int main(int argc, char **argv)
{
    int64_t size[3];
    FILE *f = argc == 3 ? fopen(argv[1], "rb") : NULL;
    if (!f || fread(size, sizeof size, 1, f) != 1) return 2;
    const size_t m = (size_t)size[0], n = (size_t)size[1], k = (size_t)size[2];
    float *x = malloc(m * k * sizeof(float)), *w = malloc(n * k * sizeof(float)), *y = malloc(m * n * sizeof(float));
    float *loss = malloc(m * sizeof(float)), *grad = malloc(m * n * sizeof(float)), *zero = calloc(m, sizeof(float));
    if (!x || !w || !y || !loss || !grad || !zero) return 2;
    if (fread(x, sizeof(float), m * k, f) != m * k || fread(w, sizeof(float), n * k, f) != n * k) return 2;
    fclose(f);
    float *dx = on_device(x, m * k), *dw = on_device(w, n * k), *dy = on_device(NULL, m * n), *dl = on_device(NULL, m);
    float *dg = on_device(NULL, m * n), *dt = on_device(zero, m), *di = on_device(zero, m);      /* zero bits: token 0 */
    void *qx = NULL, *qw = NULL;
    CHECK(cudaMalloc(&qx, zoa_mx4_size(m, k)));
    CHECK(cudaMalloc(&qw, zoa_mx4_size(n, k)));
    CHECK(zoa_mx4_quantize(dx, ZOA_F32, m, k, k, qx, NULL, NULL));
    CHECK(zoa_mx4_quantize(dw, ZOA_F32, n, k, k, qw, NULL, NULL));
    CHECK(zoa_mx4_matmul(qx, qw, m, n, k, dy, ZOA_F32, n, NULL));
    zoa_distill_args args = {0};
    args.logits = dy;
    args.index = (const int32_t *)di;
    args.teacher = dt;
    args.rows = m;
    args.vocab = n;
    args.top = 1;
    args.ld_logits = n;
    args.dtype = ZOA_F32;
    args.temperature = args.soft_weight = 1.0f;
    CHECK(zoa_distill_topk(&args, dl, NULL, dg, n, NULL));
    if (zoa_mx4_matmul(qx, qw, m, n, k, dy, ZOA_F32, n - 1, NULL) != ZOA_ERR_ARG) return 3;
    CHECK(zoa_ops_check_device());
    CHECK(cudaMemcpy(y, dy, m * n * sizeof(float), cudaMemcpyDeviceToHost));
    CHECK(cudaMemcpy(loss, dl, m * sizeof(float), cudaMemcpyDeviceToHost));
    CHECK(cudaMemcpy(grad, dg, m * n * sizeof(float), cudaMemcpyDeviceToHost));
    f = fopen(argv[2], "wb");
    if (!f || fwrite(y, sizeof(float), m * n, f) != m * n || fwrite(loss, sizeof(float), m, f) != m || fwrite(grad, sizeof(float), m * n, f) != m * n)
        return 2;
    return fclose(f) ? 2 : 0;
}
