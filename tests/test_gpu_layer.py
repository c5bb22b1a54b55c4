"""layer.MoELayer: the norms, the router and the experts together, on both sides of the few-token limit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def setup():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding as B
    from paper_2608_13057_b200.layer import MoELayer
    g = torch.Generator().manual_seed(11)
    E, G, R, k, d, f = 12, 7, 2, 3, 256, 384
    w13, s13, ref13 = _fp8(torch.randn(G, 2 * f, d, generator=g) * 0.05)
    w2, s2, ref2 = _fp8(torch.randn(G, d, f, generator=g) * 0.05)
    shape = B.make_shape(1, k, E, G, R, d, f, 128)
    packed = torch.empty(B.tempo_packed_weight_bytes(shape), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.tempo_pack_weights(shape, w13.cuda(), s13.cuda(), w2.cuda(), s2.cuda(), packed, st)
    rmap = torch.full((E, R), -1, dtype=torch.int32)
    rmap[:6, 0] = torch.arange(6, dtype=torch.int32)
    rmap[2, 1] = 6                                             # a second copy of expert 2: the same weights
    w13[6], s13[6], ref13[6], w2[6], s2[6], ref2[6] = w13[2], s13[2], ref13[2], w2[2], s2[2], ref2[2]
    B.tempo_pack_weights(shape, w13.cuda(), s13.cuda(), w2.cuda(), s2.cuda(), packed, st)
    # router weights and inputs far from ties, so that 64-bit logits choose the same experts
    w_router = (torch.randn(E, d, generator=g) * 0.2).bfloat16()
    norms = [(1 + 0.1 * torch.randn(d, generator=g)).bfloat16() for _ in range(3)]
    gate = torch.rand(d, generator=g) + 0.5
    layer = MoELayer(300, k, G, f, w_router.cuda(), rmap.cuda(), packed, norms[0].cuda(), post_w=norms[1].cuda(),
                     next_w=norms[2].cuda(), gate=gate.cuda(), r_scale=0.9, y_scale=1.1)
    return B, layer, dict(w13=ref13, w2=ref2, rmap=rmap, w_router=w_router, norms=norms, gate=gate, k=k, f=f)


def _fp8(w):
    G, n, k = w.shape
    blk = w.view(G, n // 128, 128, k // 128, 128)
    s = torch.exp2(torch.ceil(torch.log2(blk.abs().amax(dim=(2, 4), keepdim=True) / 448)))
    q = (blk / s).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).reshape(G, n, k).clone(), s.reshape(G, n // 128, k // 128).contiguous(), \
        (q.double() * s.double()).reshape(G, n, k)


def definition(c, r):
    norm = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w.double()
    x = norm(r, c["norms"][0]).float().bfloat16().double()
    p = torch.softmax(x @ c["w_router"].double().t(), 1)
    w, ids = torch.topk(p, c["k"], dim=1)
    w = w / w.sum(1, keepdim=True)
    y = torch.zeros_like(x)
    for t in range(r.shape[0]):
        for j in range(c["k"]):
            slot = int(c["rmap"][int(ids[t, j]), 0])
            if slot < 0:
                continue
            gu = c["w13"][slot] @ x[t]
            h = gu[:c["f"]] * torch.sigmoid(gu[:c["f"]]) * gu[c["f"]:]
            y[t] += w[t, j] * (c["w2"][slot] @ h)
    r2 = 0.9 * r + 1.1 * c["gate"].double() * norm(y, c["norms"][1])
    return r2, norm(r2, c["norms"][2])


@pytest.mark.parametrize("T", [1, 7, 64, 65, 300])
def test_layer_matches_the_definition(setup, T):
    """Relative error of the stream's update: three bf16 roundings on its way (x, y, x'; 1.7e-3 each, root mean square) and the
    split of H add up to 3e-3 with the few-token kernel, 5e-3 is granted; 6e-2 with the block, whose 8-bit activations are off
    by up to 2^-4 each."""
    B, layer, c = setup
    layer.status.zero_()
    r = torch.randn(T, layer.d, generator=torch.Generator().manual_seed(T))
    out, x = torch.empty(T, layer.d, device="cuda"), torch.empty(T, layer.d, dtype=torch.bfloat16, device="cuda")
    layer.forward(r.cuda(), out, x)
    torch.cuda.synchronize()
    assert int(layer.status.item()) == 0
    ref, ref_x = definition(c, r.double())
    tol = 5e-3 if T <= 64 else 6e-2
    upd, ref_upd = out.double().cpu() - 0.9 * r.double(), ref - 0.9 * r.double()
    assert float((upd - ref_upd).norm() / ref_upd.norm()) < tol
    assert float((x.double().cpu() - ref_x).norm() / ref_x.norm()) < tol


def test_in_place_and_too_many_tokens(setup):
    B, layer, c = setup
    r = torch.randn(9, layer.d, generator=torch.Generator().manual_seed(5)).cuda()
    out = layer.forward(r, torch.empty_like(r))
    same = r.clone()
    layer.forward(same, same)
    torch.cuda.synchronize()
    assert torch.equal(out, same)
    with pytest.raises(B.TempoError):
        layer.forward(torch.zeros(301, layer.d, device="cuda"), torch.zeros(301, layer.d, device="cuda"))
