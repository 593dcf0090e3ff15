/*
 * A plain C user of the feed-forward calls of include/dpo.h: residual and norm, the gated
 * block, their backward passes with the activations between kept in 8 bits.
 *
 *   ffn_consumer <in> <out>
 *   in:  int64 tokens, dim, hidden; bf16 x, residual [tokens][dim], w_norm [dim],
 *        w_gate, w_up [hidden][dim], w_down [dim][hidden], dout [tokens][dim]
 *   out: bf16 out, dx [tokens][dim], float dw_norm [dim], float dw_gate, dw_up, dw_down as
 *        the weights, uint32 status, int32 code of a refused call, char[128] its message
 *
 * Exit status 0 on success; otherwise a message on stderr and status 1.
 */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <cuda_runtime.h>

#include "dpo.h"

static void die(const char *what, const char *detail)
{
    fprintf(stderr, "ffn_consumer: %s: %s\n", what, detail ? detail : "");
    exit(1);
}

static void check_cuda(cudaError_t e, const char *what)
{
    if (e != cudaSuccess)
        die(what, cudaGetErrorString(e));
}

static void check_dpo(int rc, const char *what)
{
    if (rc != DPO_OK)
        die(what, dpo_last_error(NULL));
}

static void *dev_alloc(int64_t bytes)
{
    void *p = NULL;
    check_cuda(cudaMalloc(&p, (size_t)bytes), "cudaMalloc");
    return p;
}

static void *dev_read(FILE *f, int64_t bytes)
{
    void *host = malloc((size_t)bytes), *p = dev_alloc(bytes);
    if (host == NULL || fread(host, 1, (size_t)bytes, f) != (size_t)bytes)
        die("input", "short read");
    check_cuda(cudaMemcpy(p, host, (size_t)bytes, cudaMemcpyHostToDevice), "copy in");
    free(host);
    return p;
}

static void dev_write(FILE *f, const void *p, int64_t bytes)
{
    void *host = malloc((size_t)bytes);
    if (host == NULL)
        die("output", "memory");
    check_cuda(cudaMemcpy(host, p, (size_t)bytes, cudaMemcpyDeviceToHost), "copy out");
    if (fwrite(host, 1, (size_t)bytes, f) != (size_t)bytes)
        die("output", "short write");
    free(host);
}

static dpo_packed8 packed(int64_t rows, int64_t cols)
{
    dpo_packed8 p;
    p.ld_codes = (cols + 15) / 16 * 16;
    p.ld_scales = (cols + DPO_PACK8_GROUP - 1) / DPO_PACK8_GROUP;
    p.codes = dev_alloc(rows * p.ld_codes);
    p.scales = dev_alloc(rows * p.ld_scales);
    return p;
}

int main(int argc, char **argv)
{
    if (argc != 3)
        die("usage", "ffn_consumer <in> <out>");
    FILE *in = fopen(argv[1], "rb"), *out = fopen(argv[2], "wb");
    if (in == NULL || out == NULL)
        die("files", argv[1]);
    int64_t size[3];
    if (fread(size, sizeof size[0], 3, in) != 3)
        die("input", "short read");
    const int64_t T = size[0], D = size[1], F = size[2];
    void *x = dev_read(in, T * D * 2), *residual = dev_read(in, T * D * 2);
    void *w_norm = dev_read(in, D * 2), *w_gate = dev_read(in, F * D * 2);
    void *w_up = dev_read(in, F * D * 2), *w_down = dev_read(in, D * F * 2);
    void *dout = dev_read(in, T * D * 2);
    cudaStream_t stream;
    check_cuda(cudaStreamCreate(&stream), "stream");

    dpo_rmsnorm_args n;
    memset(&n, 0, sizeof n);
    n.x = x;
    n.residual = residual;
    n.weight = w_norm;
    n.y = dev_alloc(T * D * 2);
    n.rstd = dev_alloc(T * 4);
    n.x8 = packed(T, D);
    n.rows = T;
    n.cols = n.ld_x = n.ld_residual = n.ld_y = D;
    n.eps = 1e-5f;
    n.dtype = n.weight_dtype = DPO_BF16;
    check_dpo(dpo_rmsnorm(&n, stream), "dpo_rmsnorm");

    int64_t forward = 0, backward = 0, sums = 0;
    check_dpo(dpo_ffn_workspace(T, D, F, 1, &forward, &backward), "dpo_ffn_workspace");
    check_dpo(dpo_rmsnorm_workspace(T, D, &sums), "dpo_rmsnorm_workspace");
    dpo_ffn_args f;
    memset(&f, 0, sizeof f);
    f.x = n.y;
    f.w_gate = w_gate;
    f.w_up = w_up;
    f.w_down = w_down;
    f.out = dev_alloc(T * D * 2);
    f.gate8 = packed(T, F);
    f.up8 = packed(T, F);
    f.tokens = T;
    f.dim = f.ld_x = f.ld_out = D;
    f.hidden = F;
    f.act = DPO_ACT_SILU;
    f.keep = DPO_KEEP_8BIT;
    f.workspace = dev_alloc(forward);
    f.workspace_bytes = forward;
    check_dpo(dpo_ffn_forward(&f, stream), "dpo_ffn_forward");

    dpo_ffn_backward_args b;
    memset(&b, 0, sizeof b);
    b.dout = dout;
    b.x8 = n.x8;
    b.gain = w_norm;
    b.gain_dtype = DPO_BF16;
    b.w_gate = w_gate;
    b.w_up = w_up;
    b.w_down = w_down;
    b.gate8 = f.gate8;
    b.up8 = f.up8;
    b.dx = dev_alloc(T * D * 2);
    b.dw_gate = dev_alloc(F * D * 4);
    b.dw_up = dev_alloc(F * D * 4);
    b.dw_down = dev_alloc(D * F * 4);
    b.tokens = T;
    b.dim = b.ld_dout = b.ld_dx = D;
    b.hidden = F;
    b.act = f.act;
    b.keep = f.keep;
    b.grad_dtype = DPO_F32;
    b.workspace = dev_alloc(backward);
    b.workspace_bytes = backward;
    check_dpo(dpo_ffn_backward(&b, stream), "dpo_ffn_backward");

    dpo_rmsnorm_backward_args m;
    memset(&m, 0, sizeof m);
    m.dy = b.dx;
    m.x8 = n.x8;
    m.rstd = n.rstd;
    m.weight = w_norm;
    m.dh = dout;
    m.dx = dev_alloc(T * D * 2);
    m.dweight = dev_alloc(D * 4);
    m.rows = T;
    m.cols = m.ld_dy = m.ld_dh = m.ld_dx = D;
    m.dtype = m.weight_dtype = DPO_BF16;
    m.dweight_dtype = DPO_F32;
    m.workspace = dev_alloc(sums);
    m.workspace_bytes = sums;
    check_dpo(dpo_rmsnorm_backward(&m, stream), "dpo_rmsnorm_backward");
    check_cuda(cudaStreamSynchronize(stream), "synchronize");

    dev_write(out, f.out, T * D * 2);
    dev_write(out, m.dx, T * D * 2);
    dev_write(out, m.dweight, D * 4);
    dev_write(out, b.dw_gate, F * D * 4);
    dev_write(out, b.dw_up, F * D * 4);
    dev_write(out, b.dw_down, D * F * 4);
    uint32_t status = 1;
    check_dpo(dpo_ffn_get_status(&status), "dpo_ffn_get_status");
    f.hidden = F + 1;
    const int32_t code = dpo_ffn_forward(&f, stream);
    char message[128] = {0};
    strncpy(message, dpo_last_error(NULL), sizeof message - 1);
    if (fwrite(&status, 4, 1, out) != 1 || fwrite(&code, 4, 1, out) != 1 ||
        fwrite(message, sizeof message, 1, out) != 1 || fclose(out) != 0)
        die("output", "short write");
    return 0;
}
