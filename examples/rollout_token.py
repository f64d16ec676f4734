"""A rollout's first token right after a weight sync, on the library's kernels.

A trainer's MoE parameters (a scaled-down Qwen3 shape, random weights) are packed
into buckets, pulled and unpacked into the rollout's tensors
(``rr_pack``, ``rr_unpack_verify``).  The rollout then quantises its dense
matrices to 4 bits (``rr_quantize``) and runs one token step for a batch of
one-token prompts: fused QKV, output projection and logits with ``rr_matvec``,
the experts with ``rr_moe`` on the stacked tensors as the sync left them (or, with
``--experts 4bit``, quantised as well).  With one position, attention is the
identity on the values and the rotation is by zero, so the products are the
whole step but for the norms, which torch does.

    python examples/rollout_token.py [--tokens 4] [--experts 16bit|4bit]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2512_22492_gb300 as rr  # noqa: E402
import synth  # noqa: E402

TOP_K, EPS = 2, 1e-6


def norm(x, weight):
    v = x.float()
    return (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * weight.float()).to(x.dtype)


def sync(workload):
    """One weight sync; the rollout's tensors by name."""
    shape = workload.shape
    manifest, src, dst = rr.qwen3_sync(shape, "f32", n_shards=4, tp=1)
    plan = rr.rr_plan_create(manifest, src, dst, workload.bucket_bytes)
    gen = torch.Generator("cuda").manual_seed(workload.seed)
    flat = torch.zeros(plan.n_shards * plan.shard_bytes // 4, device="cuda")
    for p, off in zip(manifest, plan.param_flat_offset):
        n = 1
        for d in p.shape:
            n *= d
        v = 0.05 * torch.randn(n, device="cuda", generator=gen)
        flat[off // 4:off // 4 + n] = 1 + v if p.name.endswith("norm.weight") else v
    shards = list(flat.view(plan.n_shards, -1))
    buckets = torch.empty(plan.n_buckets, plan.bucket_bytes, dtype=torch.uint8, device="cuda")
    checksums = torch.empty(plan.n_buckets, dtype=torch.int64, device="cuda")
    tensors = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in plan.tensor_numel]
    rr.rr_pack(plan, shards, buckets, checksums)
    n_bad, _ = rr.rr_unpack_verify(plan, buckets, checksums, tensors)
    if n_bad:
        raise RuntimeError(f"{n_bad} buckets do not verify")
    return dict(zip(plan.tensor_names, tensors))


class Rollout:
    """The rollout's side: tensors as synced, matrices quantised once per sync."""

    def __init__(self, shape, tensors, max_tokens, experts="16bit", group=32):
        self.shape, self.t = shape, tensors
        h, q, kv = shape.hidden, shape.n_q * shape.head_dim, shape.n_kv * shape.head_dim
        self.kv, self.q = kv, q

        def packed(name, rows, cols, **kw):
            m = rr.Quantized(rows, cols, group, **kw)
            rr.rr_quantize(m, tensors[name])
            return m

        self.layers = []
        for i in range(shape.layers):
            at = f"layers.{i}."
            E, m = shape.n_experts, shape.moe_intermediate
            if experts == "4bit":
                w13 = packed(at + "experts.w13", 2 * m, h, pair=True, count=E)
                w2 = packed(at + "experts.w2", h, m, count=E)
            else:
                w13 = tensors[at + "experts.w13"].view(E, 2 * m, h)
                w2 = tensors[at + "experts.w2"].view(E, h, m)
            moe = rr.MoeLayer(tensors[at + "router"].view(E, h), w13, w2, TOP_K)
            self.layers.append((packed(at + "qkv_proj", q + 2 * kv, h),
                                packed(at + "o_proj", h, q), moe,
                                tensors[at + "input_layernorm"],
                                tensors[at + "post_attention_layernorm"]))
        self.lm_head = packed("lm_head", shape.vocab, h)
        self.workspace = rr.MoeWorkspace(self.layers[0][2], max_tokens)

    def step(self, prompt):
        """Logits [tokens, vocab] (float32) for one-token prompts."""
        s, n = self.shape, prompt.numel()
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")
        x = self.t["embed_tokens"].view(s.vocab, s.hidden)[prompt]
        for qkv_proj, o_proj, moe, norm1, norm2 in self.layers:
            qkv, attn, y = new(n, self.q + 2 * self.kv), new(n, s.hidden), new(n, s.hidden)
            rr.rr_matvec(qkv_proj, norm(x, norm1), qkv)
            # One position: every head's output is its group's value.
            v = qkv[:, self.q + self.kv:].view(n, s.n_kv, 1, s.head_dim)
            heads = v.expand(n, s.n_kv, s.n_q // s.n_kv, s.head_dim).reshape(n, self.q)
            rr.rr_matvec(o_proj, heads, attn)
            x = x + attn
            rr.rr_moe(moe, norm(x, norm2), y, self.workspace)
            x = x + y
        logits = new(n, s.vocab, dtype=torch.float32)
        rr.rr_matvec(self.lm_head, norm(x, self.t["norm"]), logits)
        return logits


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4, help="prompts of one token (1..16)")
    ap.add_argument("--experts", choices=("16bit", "4bit"), default="16bit")
    args = ap.parse_args()
    workload = synth.TEST_WORKLOADS["tiny-moe"]
    rollout = Rollout(workload.shape, sync(workload), args.tokens, args.experts)
    prompt = torch.arange(args.tokens, device="cuda") * 7 % workload.shape.vocab
    logits = rollout.step(prompt)
    for layer in rollout.layers:
        rr.rr_moe_check(layer[2], rollout.workspace)
    print("prompt", prompt.tolist(), "next", logits.argmax(-1).tolist())


if __name__ == "__main__":
    main()
