"""The token-step example: a sync, then a one-token step on 4-bit matrices and the
experts as synced, against the same step in plain 64-bit torch on the values that
the matrices stand for."""
import pytest
import torch

import synth
from tests import _products as P

pytestmark = pytest.mark.gpu


def plain_step(shape, t, prompt, experts, group, top_k, eps):
    """Norms, products and residuals as the example rounds them (bfloat16 between
    calls), each product in 64 bits."""
    bf = torch.bfloat16

    def mat(name, rows, cols):
        w = t[name].view(rows, cols)
        return P.values(*P.quantize(w, group), group)

    def norm(x, w):
        v = x.float()
        return (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + eps) * w.float()).to(bf)

    h, q, kv = shape.hidden, shape.n_q * shape.head_dim, shape.n_kv * shape.head_dim
    E, m, n = shape.n_experts, shape.moe_intermediate, prompt.numel()
    x = t["embed_tokens"].view(shape.vocab, h)[prompt]
    for i in range(shape.layers):
        at = f"layers.{i}."
        qkv = (norm(x, t[at + "input_layernorm"]).double() @ mat(at + "qkv_proj", q + 2 * kv, h).T).to(bf)
        v = qkv[:, q + kv:].view(n, shape.n_kv, 1, shape.head_dim)
        heads = v.expand(n, shape.n_kv, shape.n_q // shape.n_kv, shape.head_dim).reshape(n, q)
        x = x + (heads.double() @ mat(at + "o_proj", h, q).T).to(bf)
        y = norm(x, t[at + "post_attention_layernorm"])
        w13, w2 = t[at + "experts.w13"].view(E, 2 * m, h), t[at + "experts.w2"].view(E, h, m)
        if experts == "4bit":
            w13 = torch.stack([P.values(*P.quantize(w, group), group) for w in w13])
            w2 = torch.stack([P.values(*P.quantize(w, group), group) for w in w2])
        ids, c = P.route(y, t[at + "router"].view(E, h), top_k, True)
        out, _ = P.moe(y, ids, c, w13.double(), w2.double(), 0, "bf16")
        x = x + out.to(bf)
    return norm(x, t["norm"]).double() @ mat("lm_head", shape.vocab, h).T


@pytest.mark.parametrize("experts", ["16bit", "4bit"])
def test_example_against_plain_torch(experts):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "rollout_token.py")
    spec = importlib.util.spec_from_file_location("rollout_token", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    w = synth.TEST_WORKLOADS["tiny-moe"]
    tensors = ex.sync(w)
    rollout = ex.Rollout(w.shape, tensors, 5, experts)
    prompt = torch.tensor([0, 3, 77, 200, 511], device="cuda")
    got = rollout.step(prompt).cpu().double()
    host = {k: v.cpu() for k, v in tensors.items()}
    want = plain_step(w.shape, host, prompt.cpu(), experts, 32, ex.TOP_K, ex.EPS)
    # The two agree up to what one bfloat16 rounding that falls to the other side
    # brings about downstream: 2^-8 of a value in each of the 2 x 4 rounded steps
    # and the last norm, which the products pass on about as they are.
    rel = (got - want).norm() / want.norm()
    assert rel < 9 * 2.0 ** -8
    again = rollout.step(prompt).cpu().double()
    assert torch.equal(got, again)
