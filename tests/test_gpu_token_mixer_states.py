"""The block of the sequence operators over sequences that continue earlier ones: its gradients, to which the states that they began with are constants, against automatic
differentiation of plain operations in 64 bits, and the states that it hands on."""
import pytest
import torch

import gpu_util as gu

pytestmark = pytest.mark.gpu


def _plain(p, x, residual, bounds, rows, h0):
    """The block in 64 bits, its sequences behind the rows of the convolution and the states of the scan that they are given: (hidden, residual, rows, states)."""
    R = p["w_dt"].shape[0]
    C, N = p["A_log"].shape
    K = p["conv_w"].shape[0]
    s = x + residual
    xz = torch.nn.functional.layer_norm(s, s.shape[1:], p["norm_w"], p["norm_b"], 1e-5) @ p["w_in"]
    xi, z = xz[:, :C], xz[:, C:]
    outs, new_rows, new_h = [], [], []
    for i, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        line = torch.cat([rows[i], xi[lo:hi]])
        u = torch.nn.functional.silu(sum(p["conv_w"][k] * line[k:k + hi - lo] for k in range(K)) + p["conv_b"])
        proj = u @ p["w_x"]
        delta = torch.nn.functional.softplus(proj[:, :R] @ p["w_dt"] + p["dt_bias"])
        B, Cm = proj[:, R:R + N], proj[:, R + N:]
        h = h0[i]
        for t in range(hi - lo):
            h = torch.exp(delta[t][:, None] * -torch.exp(p["A_log"])) * h + (delta[t] * u[t])[:, None] * B[t]
            outs.append((h @ Cm[t] + p["D"] * u[t]) * torch.nn.functional.silu(z[lo + t]))
        new_rows.append(line[hi - lo:])
        new_h.append(h)
    return torch.stack(outs) @ p["w_out"], s, torch.stack(new_rows), torch.stack(new_h)


@pytest.mark.parametrize("bounds,packed", [([0, 9, 9, 41], True), ([0, 18, 36], False)])
def test_gradients_of_a_block_that_continues(gpu_lib, bounds, packed):
    from paper_1803_09926_amd.token_mixer import TokenMixer
    torch.manual_seed(8)
    M, S, T = 32, len(bounds) - 1, bounds[-1]
    block = TokenMixer(M, states=5, dtype=torch.float32, seed=6)
    x, residual, dh, dr = (torch.randn(T, M) for _ in range(4))
    rows, h = torch.randn(S, block.K - 1, block.C), torch.randn(S, block.C, block.N)
    states = (rows.cuda(), h.cuda())
    starts = torch.tensor(bounds, dtype=torch.int32, device="cuda") if packed else None
    hidden, total = block.forward(x.cuda(), residual.cuda(), starts, S, states=states, keep=True)
    dx, grads = block.backward(dh.cuda(), dr.cuda())
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in block.p.items()}
    x64 = x.double().requires_grad_()
    want, s, new_rows, new_h = _plain(p, x64, residual.double(), bounds, rows.double(), h.double())
    ((want * dh).sum() + (s * dr).sum()).backward()
    # fp32 products of up to 64 terms in a row of four, each within about 1e-6 of its size: 2e-5 for the chain, 5e-5 for sums over tokens behind it
    gu.assert_close(gu.to_host(hidden), want.detach().numpy(), 2e-5, "hidden")
    gu.assert_close(gu.to_host(states[0]), new_rows.detach().numpy(), 2e-5, "the convolution's rows")
    gu.assert_close(gu.to_host(states[1]), new_h.detach().numpy(), 2e-5, "the scan's states")
    gu.assert_close(gu.to_host(dx), x64.grad.numpy(), 2e-5, "dx")
    for k in p:
        gu.assert_close(gu.to_host(grads[k]), p[k].grad.numpy(), 5e-5, k)


def test_calls_on_two_streams_have_workspaces_of_their_own(gpu_lib, monkeypatch):
    from paper_1803_09926_amd import token_mixer
    held = []

    def recorded(call):
        def run(*args, **named):
            held.extend(a for a in args if isinstance(a, torch.Tensor) and a.dtype == torch.uint8)
            return call(*args, **named)
        return run
    for name in ("sscan_fwd", "sscan_bwd", "cconv_bwd", "lnorm_bwd"):
        monkeypatch.setattr(token_mixer.dw, name, recorded(getattr(token_mixer.dw, name)))
    block, T = token_mixer.TokenMixer(32, dtype=torch.float32), 400
    x, dh = torch.randn(T, 32, device="cuda"), torch.randn(T, 32, device="cuda")
    torch.cuda.synchronize()
    side, counts = torch.cuda.Stream(), []
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            block.forward(x, keep=True)
            block.backward(dh)
        counts.append(len(held))
    torch.cuda.synchronize()
    first, second = ({t.data_ptr() for t in held[a:b] if t.numel() > 16} for a, b in ((0, counts[0]), (counts[0], counts[1])))
    assert first and second and not first & second


def test_two_forwards_before_a_backward(gpu_lib):
    from paper_1803_09926_amd.token_mixer import TokenMixer
    block = TokenMixer(32, dtype=torch.float32)
    a, b, da, db = (torch.randn(50, 32, device="cuda") for _ in range(4))
    with pytest.raises(RuntimeError, match="came before"):
        block.backward(da)

    def alone(x, d):
        block.forward(x, keep=True)
        dx, g = block.backward(d)
        again, _ = block.backward(d)                     # (as often as one likes)
        assert torch.equal(dx, again)
        return dx, g
    want_a, want_b = alone(a, da), alone(b, db)
    block.forward(a, keep=True)
    kept = block.kept
    block.forward(b, keep=True)
    got_b = block.backward(db)
    with pytest.raises(RuntimeError, match="replaced"):  # not the second one's once more
        block.backward(da)
    got_a = block.backward(da, kept=kept)
    for got, want in ((got_a, want_a), (got_b, want_b)):
        assert torch.equal(got[0], want[0]) and all(torch.equal(got[1][k], want[1][k]) for k in want[1])
