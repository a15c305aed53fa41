"""A layer of experts whose weights are BitStack stacks, run in 8-bit floating point: every expert's two weights are restored from the blocks that
are loaded, brought to 8 bits, and multiplied with the rows of the tokens routed to it.

    python examples/expert_layer.py        (needs an MI355X)
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_23918_amd as B  # noqa: E402


class ExpertLayer:
    """y = sum over a token's experts e of p_e  W2_e (g / (1 + exp(-g)) u),  (g, u) = W1_e x.

    router: [experts, hidden]; w1, w2: (q, scales) of all experts, [experts, 2 width, hidden] (gates above values) and [experts, hidden, width].

    A few tokens go through the layer in one call, which takes activations as they are (their products, of a block of 128 columns before its scale, have to be
    finite: up to 1e33); others through four, which bring them to 8 bits, some 4 % of y's norm.  So y changes by as much where the number of tokens passes from one to
    the other."""

    def __init__(self, router, w1, w2, top_k: int):
        self.router, self.w1, self.w2, self.top_k = router, w1, w2, top_k

    @classmethod
    def from_stacks(cls, router, stacks1, stacks2, n_loaded: int, top_k: int):
        """the weights as the first n_loaded blocks of every expert's stacks give them; one fp16 scratch for all"""
        def all_of(stacks):
            out, inn, e = stacks[0].out, stacks[0].inn, len(stacks)
            scratch = torch.empty((out, inn), dtype=torch.float16, device=router.device)
            q = torch.empty((e, out, -(-inn // 128) * 128), dtype=torch.float8_e4m3fn, device=router.device)[:, :, :inn]
            scales = torch.empty((e, -(-out // 128), -(-inn // 128)), dtype=torch.float8_e8m0fnu, device=router.device)
            for i, stack in enumerate(stacks):   # each where it will lie among the others
                stack.restore_weight_f8(n_loaded, w_dense=scratch, out=(q[i], scales[i]))
            return q, scales
        return cls(router, all_of(stacks1), all_of(stacks2), top_k)

    def in_one_call(self, x) -> bool:
        """Does the layer's one call take these tokens, and in less time than the four?  On an MI355X, one call and four: 64 experts of 4096 x 1024, six chosen, bf16, 16 tokens
        126 us and 152, 64 tokens 158 and 186; eight of 4096 x 14336, two chosen, bf16, 16 tokens (four to an expert) 254 and 257, 64 tokens 293 and 269, fp32, one token 89 and
        89, 16 tokens 324 and 309; 384 of 7168 x 2048, eight chosen, bf16, 16 tokens 914 and 894.  Where the weights are small (four of 512 x 768, 64 tokens, bf16: 24 and 52)
        four calls take the host longer than the GPU."""
        (experts, rows, hidden), tokens = self.w1[0].shape, x.shape[0]
        if tokens > 64 or hidden < 8 or rows > 2**16 or self.w1[0].stride(0) >= 2**32:   # (the call's limits; width: 2 GiB of h)
            return False
        wide = x.dtype is torch.float32 and hidden > 2048
        to_an_expert = tokens * self.top_k / experts
        small = 3 * rows // 2 * hidden * experts * x.element_size() <= 2**27
        return small or (experts <= 256 and to_an_expert <= (0.5 if wide else 8))

    def __call__(self, x):
        logits = x.float() @ self.router.T
        if self.in_one_call(x):
            return B.expert_layer_f8(x, logits, self.w1, self.w2, self.top_k)
        r = B.route(logits, self.top_k)
        h = B.grouped_linear_f8(x, *self.w1, r.offsets, r.rows)              # a row for each (token, expert), sorted by expert
        y = B.grouped_linear_f8(h, *self.w2, r.offsets, gated=True)
        return B.combine(y, r.slots, r.weights)


def plain(layer, x):
    """the same in fp32, with the weights' 8-bit values and without bringing the activations to 8 bits"""
    def values(w):
        q, s = w
        return q.float() * s.float().repeat_interleave(128, 1)[:, : q.shape[1]].repeat_interleave(128, 2)[:, :, : q.shape[2]]
    x = x.float()
    best, experts = torch.topk(x @ layer.router.T, layer.top_k)
    p, w1, w2, y = torch.softmax(best, 1), values(layer.w1), values(layer.w2), torch.zeros_like(x)
    for e in range(w1.shape[0]):
        t, j = torch.nonzero(experts == e, as_tuple=True)
        g, u = (x[t] @ w1[e].T).chunk(2, 1)
        y.index_add_(0, t, p[t, j][:, None] * ((g / (1 + torch.exp(-g)) * u) @ w2[e].T))
    return y


def make(hidden=512, width=768, experts=4, blocks=3, top_k=2, seed=0):
    """stacks decomposed on the device from random weights"""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ones = lambda n: torch.ones(n).numpy()
    stack = lambda out, inn: B.PackedStack.from_dense(torch.randn((out, inn), generator=g, device="cuda") * inn**-0.5, ones(inn), n=blocks, iterations=4)
    router = torch.randn((experts, hidden), generator=g, device="cuda") * hidden**-0.5
    return ExpertLayer.from_stacks(router, [stack(2 * width, hidden) for _ in range(experts)], [stack(hidden, width) for _ in range(experts)], blocks, top_k)


if __name__ == "__main__":
    layer = make()
    for tokens in (1, 57, 2048):
        x = torch.randn((tokens, 512), device="cuda").to(torch.bfloat16)
        y, want = layer(x).float(), plain(layer, x)
        print(f"{tokens} tokens: relative difference to fp32 activations {((y - want).norm() / want.norm()).item():.3f}")
