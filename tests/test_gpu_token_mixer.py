"""The block that runs the sequence operators together: its gradients against automatic differentiation of plain operations in 64 bits, token by token against a
prompt read at once, and a training run."""
import pytest
import torch

import gpu_util as gu

pytestmark = pytest.mark.gpu


def _plain(p, x, residual, bounds):
    """The block in 64 bits: (hidden, residual) of packed sequences."""
    R = p["w_dt"].shape[0]
    C, N = p["A_log"].shape
    K = p["conv_w"].shape[0]
    s = x + residual
    normed = torch.nn.functional.layer_norm(s, s.shape[1:], p["norm_w"], p["norm_b"], 1e-5)
    xz = normed @ p["w_in"]
    xi, z = xz[:, :C], xz[:, C:]
    outs = []
    for lo, hi in zip(bounds[:-1], bounds[1:]):
        line = torch.cat([torch.zeros(K - 1, C, dtype=x.dtype), xi[lo:hi]])
        u = torch.nn.functional.silu(sum(p["conv_w"][k] * line[k:k + hi - lo] for k in range(K)) + p["conv_b"])
        proj = u @ p["w_x"]
        delta = torch.nn.functional.softplus(proj[:, :R] @ p["w_dt"] + p["dt_bias"])
        B, Cm = proj[:, R:R + N], proj[:, R + N:]
        h = torch.zeros(C, N, dtype=x.dtype)
        for t in range(hi - lo):
            h = torch.exp(delta[t][:, None] * -torch.exp(p["A_log"])) * h + (delta[t] * u[t])[:, None] * B[t]
            outs.append((h @ Cm[t] + p["D"] * u[t]) * torch.nn.functional.silu(z[lo + t]))
    return torch.stack(outs) @ p["w_out"], s


def test_gradients_of_a_block(gpu_lib):
    from paper_1803_09926_amd.token_mixer import TokenMixer
    torch.manual_seed(3)
    bounds, M = [0, 9, 9, 30], 32
    block = TokenMixer(M, states=5, dtype=torch.float32, seed=4)
    x, residual, dh, dr = (torch.randn(bounds[-1], M) for _ in range(4))
    starts = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    hidden, total = block.forward(x.cuda(), residual.cuda(), starts, len(bounds) - 1, keep=True)
    dx, grads = block.backward(dh.cuda(), dr.cuda())
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in block.p.items()}
    x64, r64 = x.double().requires_grad_(), residual.double()
    want, s = _plain(p, x64, r64, bounds)
    ((want * dh).sum() + (s * dr).sum()).backward()
    # fp32 products of up to 64 terms in a row of four, each within about 1e-6 of its size: 2e-5 for the chain
    gu.assert_close(gu.to_host(hidden), want.detach().numpy(), 2e-5, "hidden")
    gu.assert_close(gu.to_host(total), s.detach().numpy(), 1e-6, "residual")
    gu.assert_close(gu.to_host(dx), x64.grad.numpy(), 2e-5, "dx")
    for k in p:
        gu.assert_close(gu.to_host(grads[k]), p[k].grad.numpy(), 5e-5, k)


def test_training_and_generation(gpu_lib):
    from paper_1803_09926_amd import token_mixer
    losses, off = token_mixer.main(["--width", "128", "--tokens", "640", "--steps", "6", "--generate", "6"])
    assert losses[-1] < losses[0] and all(l == l for l in losses)
    # bf16 activations are rounded about ten times a block, to 2^-9 each, along either way
    assert off < 5e-2
