"""Compresses a model's output matrix and says what that costs.

    python examples/compress_output_matrix.py [--vocab 32768 --dim 1024 --rank 128 --tokens 4096 --steps 40]

W (vocab x dim), as in a trained model with a spectrum that falls off, is factored by the block randomized SVD, W ~ U S V^T,
and what the factors leave is kept in 8 bits with a scale for each 128 x 128 block, or in 4 bits with a scale for each 32
numbers of a row.  The loss of the model's logits H W^T is worked out without them: for W, for the factors alone (hidden states
H V S of width rank, output matrix U) and for the factors with the remainder.  Then U is repaired by distillation from the
stored top logits of W: clipped gradient steps on the divergence, whose effect the cross entropy shows.  Inputs are synthetic."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1706_07191_amd as B  # noqa: E402


def model(vocab, dim, tokens, seed, dev):
    """An output matrix, hidden states and the words that follow: drawn from the model's own distribution."""
    g = torch.Generator(device=dev).manual_seed(seed)
    r = min(vocab, dim)
    decay = torch.arange(1, r + 1, device=dev).float().pow(-0.7)
    W = (torch.randn(vocab, r, generator=g, device=dev) * decay) @ torch.randn(r, dim, generator=g, device=dev) / math.sqrt(r)
    W = W / W.pow(2).mean().sqrt() / math.sqrt(dim) * 5.0
    H = torch.randn(tokens, dim, generator=g, device=dev)
    words, top_ids, top = [], [], []
    for h in H.split(1024):
        z = h @ W.t()
        words.append(torch.multinomial(torch.softmax(z, dim=1), 1, generator=g)[:, 0])
        v, i = z.topk(64, dim=1)
        top.append(v)
        top_ids.append(i)
    return W, H, torch.cat(words), torch.cat(top_ids).contiguous(), torch.cat(top).contiguous()


def factors(W, rank, seed):
    """U (vocab x rank), S, V^T of W, by the library."""
    vocab, dim = W.shape
    p = min(16, min(vocab, dim) - rank)
    Omega = B.brsvd_philox_normal(seed, dim, rank + p, device=W.device)
    handle = B.brsvd_create(B.make_params(vocab, dim, rank, p, 1))
    try:
        U, S, Vt, _ = B.brsvd_run(handle, W, Omega)
    finally:
        B.brsvd_destroy(handle)
    return U[:, :rank].contiguous(), S[:rank], Vt[:rank].contiguous()


def mean_loss(H, W, words):
    return float(B.brsvd_xent_forward(H.bfloat16(), W.bfloat16(), words)[0].mean())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--vocab", type=int, default=32768)
    ap.add_argument("--dim", type=int, default=1024)
    ap.add_argument("--rank", type=int, default=128)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--temperature", type=float, default=1.0)
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    W, H, words, ids, top = model(a.vocab, a.dim, a.tokens, 1, dev)
    said = {"whole": mean_loss(H, W, words)}

    U, S, Vt = factors(W, a.rank, 2)
    narrow = (H @ Vt.t()) * S                                   # H V S: what multiplies U
    said["factors"] = mean_loss(narrow, U, words)

    # the remainder in 8 bits: as a product for serving, as a matrix for the loss
    Q, scales = B.brsvd_quantize_e4m3(W - (U * S) @ Vt, block_rows=128)
    kept = (U * S) @ Vt + B.brsvd_dequantize_e4m3(Q, scales, block_rows=128)
    said["factors and 8-bit remainder"] = mean_loss(H, kept, words)
    served = B.brsvd_linear_e4m3(H[:4], Q, scales) + narrow[:4] @ U.t()
    said["logits of four tokens off by"] = float((served - H[:4] @ W.t()).norm() / (H[:4] @ W.t()).norm())

    # and in 4 bits
    Q, scales = B.brsvd_quantize_e2m1(W - (U * S) @ Vt)
    said["factors and 4-bit remainder"] = mean_loss(H, (U * S) @ Vt + B.brsvd_dequantize_e2m1(Q, scales, cols=a.dim), words)
    served = B.brsvd_linear_e2m1(H[:4].bfloat16(), Q, scales).float() + narrow[:4] @ U.t()
    said["4 bits: logits off by"] = float((served - H[:4] @ W.t()).norm() / (H[:4] @ W.t()).norm())

    # distillation of the narrow model: its output matrix moves, the hidden states stay
    h, tau = narrow.bfloat16(), a.temperature
    weight = torch.full((1,), 1.0 / a.tokens, device=dev)
    M, moment, square, g = U.clone(), torch.zeros_like(U), torch.zeros_like(U), torch.empty_like(U)
    for step in range(a.steps):
        w = M.bfloat16()
        loss, lse, z = B.brsvd_distill_forward(h, w, ids, top, tau)
        if step == 0:
            said["divergence before"] = float(loss.mean())
        _, dW = B.brsvd_distill_backward(h, w, ids, top, tau, lse, z, weight, need_dH=False)
        norm = B.brsvd_grad_norm([dW])
        if step == 0:
            most = float(norm)                                  # later gradients are smaller unless something is wrong
        B.brsvd_grad_clip([dW], norm, most, out=[g])
        moment.lerp_(g, 0.1)
        square.lerp_(g * g, 0.02)
        M -= 0.02 * float(U.pow(2).mean().sqrt()) * (moment / (1 - 0.9 ** (step + 1))) / ((square / (1 - 0.98 ** (step + 1))).sqrt() + 1e-12)
    said["divergence after"] = float(B.brsvd_distill_forward(h, M.bfloat16(), ids, top, tau)[0].mean())
    said["factors, distilled"] = mean_loss(narrow, M, words)
    for name, value in said.items():
        print("%-32s %.4f" % (name, value))
    return said


if __name__ == "__main__":
    main()
