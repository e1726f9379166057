"""A small network trained in eight bits: two layers whose products run on 8-bit floating point, the first one's activation finished with its product, dropout onto a residual, and the
cross entropy of a linear last layer over a vocabulary, with every gradient.  Synthetic data, plain gradient descent:

    python examples/network_in_eight_bits.py [steps]

    u = x W1^T,  v = max(u, 0) W2^T,  h = dropout(v) + x,  loss = cross entropy of h E^T
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_09849_amd as cdl  # noqa: E402


def empty(*shape, dtype=torch.uint8):
    return torch.empty(shape, dtype=dtype, device="cuda")


class Blocks:
    """A matrix in 8-bit floating point, along its rows and along its columns."""

    def __init__(self, rows, cols, tiles=False, format=cdl.E4M3):
        self.rows, self.cols, self.tiles, self.format = rows, cols, tiles, format
        across, down = cdl.block8_pitch(cols), cdl.block8_pitch(rows)
        self.q, self.scale = empty(rows, across), empty(across // 128, down)
        self.q_t, self.scale_t = empty(cols, down), empty(down // 128, across)

    def set(self, x):
        cdl.cdl_block8_quantize(x, self.rows, self.cols, self.q, self.scale, self.q_t, self.scale_t, tiles=self.tiles, format=self.format)


class Layer:
    """y = x w^T: weights fp32 as the optimizer holds them, in tiles for the products; gradients in the wider-ranging format."""

    def __init__(self, tokens, out, into):
        self.M, self.N, self.K = tokens, out, into
        self.w, self.d_w = torch.randn(out, into, device="cuda") * into ** -0.5, empty(out, into, dtype=torch.float32)
        self.y, self.z, self.d_x = (empty(tokens, n, dtype=torch.bfloat16) for n in (out, out, into))
        self.x8, self.w8, self.g8 = Blocks(tokens, into), Blocks(out, into, tiles=True), Blocks(tokens, out, format=cdl.E5M2)
        sizes = ((tokens, into, out), (out, into, tokens))
        self.ws = empty(max(256, cdl.block8_gemm_act_workspace_bytes(tokens, out, into), *(cdl.block8_gemm_workspace_bytes(*s) for s in sizes)))

    def forward(self, x, act=cdl.ACT_NONE):
        """act(x w^T), and what the activation is of for its backward pass"""
        self.x8.set(x)
        self.w8.set(self.w)
        cdl.cdl_block8_gemm_act(self.x8.q, self.x8.scale, self.w8.q, self.w8.scale, self.M, self.N, self.K, self.y, z=None if act == cdl.ACT_NONE else self.z, act=act, ws=self.ws)
        return self.y

    def backward(self, g):
        x, w = self.x8, self.w8
        self.g8.set(g)
        cdl.cdl_block8_gemm(self.g8.q, self.g8.scale, w.q_t, w.scale_t, self.M, self.K, self.N, self.d_x, self.ws, a_format=cdl.E5M2)
        cdl.cdl_block8_gemm(self.g8.q_t, self.g8.scale_t, x.q_t, x.scale_t, self.N, self.K, self.M, self.d_w, self.ws, a_format=cdl.E5M2)
        return self.d_x


class Network:
    def __init__(self, tokens=1000, width=256, hidden=1024, vocabulary=5003, p=0.1, seed=1):
        torch.manual_seed(seed)
        self.T, self.D, self.V, self.p, self.seed = tokens, width, vocabulary, p, seed
        self.up, self.down = Layer(tokens, hidden, width), Layer(tokens, width, hidden)
        self.E = (torch.randn(vocabulary, width, device="cuda") * width ** -0.5).bfloat16()
        self.d_E = torch.empty_like(self.E)
        self.d_u = empty(tokens, hidden, dtype=torch.bfloat16)
        self.h, self.d_h, self.d_v = (empty(tokens, width, dtype=torch.bfloat16) for _ in range(3))
        self.loss, self.lse = (empty(tokens, dtype=torch.float32) for _ in range(2))
        self.d_loss = torch.full((tokens,), 1.0 / tokens, device="cuda")
        self.ws = empty(cdl.head_loss_workspace_bytes(tokens, vocabulary, width, cdl.BF16, True))

    def step(self, x, target, number):
        """Losses of the tokens, and every gradient."""
        T, D, V = self.T, self.D, self.V
        v = self.down.forward(self.up.forward(x, cdl.ACT_RELU))
        counter = number * ((T * D + 7) // 8)                 # no two steps share a part of the sequence
        cdl.cdl_dropout(v, T * D, self.p, self.seed, counter, self.h, add=x)
        cdl.cdl_head_loss_fwd(self.h, self.E, target, T, V, D, self.loss, self.lse, self.ws)
        cdl.cdl_head_loss_bwd(self.h, self.E, target, self.lse, T, V, D, self.d_h, self.d_E, self.ws, d_loss=self.d_loss)
        cdl.cdl_dropout(self.d_h, T * D, self.p, self.seed, counter, self.d_v)
        cdl.cdl_act_bwd(self.down.backward(self.d_v), T, self.up.N, cdl.ACT_RELU, d_z=self.d_u, z=self.up.z)
        self.up.backward(self.d_u)
        return self.loss

    def update(self, rate):
        for layer in (self.up, self.down):
            layer.w -= rate * layer.d_w
        self.E -= rate * self.d_E


def main(steps=40):
    network = Network()
    x = torch.randn(network.T, network.D, device="cuda").bfloat16()
    target = torch.randint(0, network.V, (network.T,), device="cuda")
    for number in range(steps):
        loss = network.step(x, target, number).mean().item()
        network.update(0.5)
        if number % 10 == 0 or number == steps - 1:
            print("step %3d  loss %.4f" % (number, loss), flush=True)


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:2]))
