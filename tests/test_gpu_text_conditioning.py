"""The operators together, as a text-conditioned video model uses them: a layer of the text encoder (attention with a relative position bias),
its states as keys and values of the cross attention, queries from the self attention over the video tokens, and the way back of the gradients
to the encoder's weights, its table and its input, against autograd in 64 bits on the CPU."""
import math

import pytest
import torch

from dense_util import bucket_map
from paper_2505_14708_amd import binding as da

pytestmark = pytest.mark.gpu


def test_encoder_layer_and_cross_attention():
    B, H, d, M = 2, 2, 64, 77
    T, fh, fw = 2, 16, 16
    N, W = T * fh * fw, H * d
    rule = (32, 128, 1, 0)
    gen = torch.Generator().manual_seed(0)

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen) * std
    X, Wqkv, Wkv = normal(B, M, W), normal(W, 3 * W, std=W ** -0.5), normal(W, 2 * W, std=W ** -0.5)
    table, video, G = normal(rule[0], H), normal(3, B, H, N, d), normal(B, H, N, d)
    lens = [M, 31]
    scale = 1.0 / 8

    # on the GPU
    x, wqkv, wkv, tab, g = X.cuda(), Wqkv.cuda(), Wkv.cuda(), table.cuda(), G.cuda()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    p0 = da.problem(B, H, T, fh, fw, d, dtype=da.DA_F32, sparsity=0.5)
    q2 = torch.empty(B, H, N, d, device="cuda")
    vid = video.cuda()
    da.da_forward(p0, vid[0], vid[1], vid[2], q2, torch.empty(da.da_workspace_size(p0), dtype=torch.uint8, device="cuda"))

    def heads(buf):                                            # [B, rows, n, H, d] -> n views [B, H, rows, d]
        return [buf[:, :, i].permute(0, 2, 1, 3) for i in range(buf.shape[2])]
    pe, rel = da.attn_problem(B, H, M, M, d, dtype=da.DA_F32, scale=scale), da.rel_bias(*rule)
    pc = da.attn_problem(B, H, N, M, d, dtype=da.DA_F32)
    se, sc = da.da_attn_sizes(pe, rel), da.da_attn_sizes(pc)
    ws = torch.empty(max(256, se.forward_ws, se.backward_ws, sc.forward_ws, sc.backward_ws), dtype=torch.uint8, device="cuda")
    qkv = (x @ wqkv).view(B, M, 3, H, d)
    states = torch.empty(B, M, 1, H, d, device="cuda")
    lse_e, lse_c = torch.empty(B, H, M, device="cuda"), torch.empty(B, H, N, device="cuda")
    (q, k, v), (s,) = heads(qkv), heads(states)
    dqkv, dstates = torch.empty_like(qkv), torch.empty_like(states)
    (dq, dk, dv), (ds,) = heads(dqkv), heads(dstates)
    lay = {m: da.layout_of(t) for m, t in dict(q=q, k=k, v=v, o=s, do=ds, dq=dq, dk=dk, dv=dv).items()}
    lay = da.attn_layouts(**lay)
    da.da_bias_attn(pe, rel, q, k, v, tab, s, ws, kv_len=n, lse=lse_e, layouts=lay)
    kv = (states.view(B, M, W) @ wkv).view(B, M, 2, H, d)
    dkv = torch.empty_like(kv)
    (ck, cv), (cdk, cdv) = heads(kv), heads(dkv)
    o, dq2 = torch.empty(B, H, N, d, device="cuda"), torch.empty(B, H, N, d, device="cuda")
    layc = da.attn_layouts(k=da.layout_of(ck), v=da.layout_of(cv), dk=da.layout_of(cdk), dv=da.layout_of(cdv))
    da.da_cross_attn(pc, q2, ck, cv, o, ws, kv_len=n, lse=lse_c, layouts=layc)
    da.da_cross_attn_bwd(pc, q2, ck, cv, o, lse_c, g, dq2, cdk, cdv, ws, kv_len=n, layouts=layc)
    dkv2 = dkv.view(B * M, 2 * W)
    dwkv = states.view(B * M, W).t() @ dkv2
    dstates.copy_((dkv2 @ wkv.t()).view(B, M, 1, H, d))
    dtab = torch.empty_like(tab)
    da.da_bias_attn_bwd(pe, rel, q, k, v, tab, s, lse_e, ds, dq, dk, dv, dtab, ws, kv_len=n, layouts=lay)
    dqkv2 = dqkv.view(B * M, 3 * W)
    got = dict(o=o, dq2=dq2, dwkv=dwkv, dtab=dtab, dwqkv=x.view(B * M, W).t() @ dqkv2, dx=(dqkv2 @ wqkv.t()).view(B, M, W))

    # autograd in float64
    r = [t.double().requires_grad_() for t in (X, Wqkv, Wkv, table, q2.cpu())]
    keep = torch.arange(M)[None, None, None, :] < torch.tensor(lens)[:, None, None, None]

    def attend(q, k, v, c, bias=0.0):
        return torch.softmax((q @ k.transpose(2, 3) * c + bias).masked_fill(~keep, -math.inf), 3) @ v
    e = (r[0] @ r[1]).view(B, M, 3, H, d).permute(2, 0, 3, 1, 4)
    st = attend(e[0], e[1], e[2], scale, r[3].t()[:, bucket_map(M, M, rule)]).permute(0, 2, 1, 3).reshape(B, M, W)
    c = (st @ r[2]).view(B, M, 2, H, d).permute(2, 0, 3, 1, 4)
    out = attend(r[4], c[0], c[1], d ** -0.5)
    (out * G.double()).sum().backward()
    want = dict(o=out.detach(), dq2=r[4].grad, dwkv=r[2].grad, dtab=r[3].grad, dwqkv=r[1].grad, dx=r[0].grad)
    # about ten float32 products and softmaxes in a row, each off by some 128 half steps of 2^-24 relative to its norm at worst
    for name, w in want.items():
        off = float((got[name].cpu().double() - w).norm() / w.norm())
        print(f"[gpu-test] {name}: {off:.2e}", flush=True)
        assert off < 10 * 128 * 2.0 ** -24, (name, off)
