"""layer.MoELayer at the sizes between its two paths: more than 16 choices per token, batches smaller than the buffers.
Tolerances as in test_gpu_layer."""
import pytest
import torch

from tests.test_gpu_layer import _fp8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


class Case:
    """A seeded layer of G local experts and its definition in 64 bits."""

    def __init__(self, B, max_tokens, k, E, G, d=256, f=256, **kw):
        from paper_2608_13057_b200.layer import MoELayer
        g = torch.Generator().manual_seed(k * 100 + E)
        self.B, self.k, self.G, self.d, self.f, self.kw = B, k, G, d, f, kw
        w13, w2 = torch.randn(G, 2 * f, d, generator=g) * 0.05, torch.randn(G, d, f, generator=g) * 0.05
        shape = B.make_shape(1, k, E, G, 1, d, f, 128)
        if kw.get("bf16"):
            self.w13, self.w2 = w13.bfloat16().double(), w2.bfloat16().double()
            packed = torch.empty(B.tempo_packed_weight_bytes_bf16(shape), dtype=torch.uint8, device="cuda")
            B.tempo_pack_weights_bf16(shape, w13.bfloat16().cuda(), w2.bfloat16().cuda(), packed)
        else:
            (q13, s13, self.w13), (q2, s2, self.w2) = _fp8(w13), _fp8(w2)
            packed = torch.empty(B.tempo_packed_weight_bytes(shape), dtype=torch.uint8, device="cuda")
            st = torch.zeros(1, dtype=torch.int32, device="cuda")
            B.tempo_pack_weights(shape, q13.cuda(), s13.cuda(), q2.cuda(), s2.cuda(), packed, st)
        rmap = torch.full((E, 1), -1, dtype=torch.int32)
        rmap[:G, 0] = torch.arange(G, dtype=torch.int32)
        self.w_router = (torch.randn(E, d, generator=g) * 0.2).bfloat16()
        self.norm_w = (1 + 0.1 * torch.randn(d, generator=g)).bfloat16()
        self.layer = MoELayer(max_tokens, k, G, f, self.w_router.cuda(), rmap.cuda(), packed, self.norm_w.cuda(),
                              **{n: v.cuda() if torch.is_tensor(v) else v for n, v in kw.items()})

    def norm(self, v, w, b):
        if w is None:
            return v
        if self.kw.get("kind"):
            v = v - v.mean(1, keepdim=True)
        v = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6) * w.double()
        return v if b is None else v + b.double()

    def definition(self, r):
        x = self.norm(r.double(), self.norm_w, self.kw.get("norm_b")).float().bfloat16().double()
        w, ids = torch.topk(torch.softmax(x @ self.w_router.double().t(), 1), self.k, dim=1)
        w = w / w.sum(1, keepdim=True)
        y = torch.zeros_like(x)
        for e in range(self.G):
            t, j = torch.nonzero(ids == e, as_tuple=True)
            if t.numel():
                gate, up = (x[t] @ self.w13[e].t()).chunk(2, 1)
                y.index_add_(0, t, (gate * torch.sigmoid(gate) * up) @ self.w2[e].t() * w[t, j][:, None])
        return self.norm(y, self.kw.get("post_w"), self.kw.get("post_b")), ids

    def check(self, T, few, seed=0):
        r = torch.randn(T, self.d, generator=torch.Generator().manual_seed(seed * 1000 + T))
        out, x = torch.empty(T, self.d, device="cuda"), torch.empty(T, self.d, dtype=torch.bfloat16, device="cuda")
        self.layer.forward(r.cuda(), out, x if "next_w" in self.kw else None)
        torch.cuda.synchronize()
        assert int(self.layer.status.item()) == 0
        ref, ids = self.definition(r)
        upd = out.double().cpu() - r.double()
        err = float((upd - ref).norm() / ref.norm())
        assert err < (5e-3 if few else 6e-2), (T, err)
        if "next_w" in self.kw:
            ref = self.norm(r.double() + ref, self.kw["next_w"], self.kw.get("next_b"))
            assert float((x.double().cpu() - ref).norm() / ref.norm()) < (5e-3 if few else 6e-2)
        return ids


@pytest.mark.parametrize("k,max_tokens,few", [(17, 64, 60), (20, 64, 51), (32, 40, 32), (32, 300, 32), (16, 64, 64)])
def test_more_than_sixteen_choices(B, k, max_tokens, few):
    """The few-token kernel takes 1024 (token, expert) pairs: fewer than 64 tokens above 16 choices each."""
    c = Case(B, max_tokens, k, 40, 24)
    for T in sorted({1, few - 1, few, min(few + 1, max_tokens), max_tokens}):
        c.check(T, T <= few)


def test_batches_smaller_than_the_buffers(B):
    """Above the few-token limit a batch of T rows runs as T rows: what lies behind them is not written."""
    c = Case(B, 1200, 3, 12, 7)
    for T in (1200, 65, 300, 1199, 70, 66):
        c.layer.y.fill_(float("nan"))
        c.check(T, False)
        assert torch.isnan(c.layer.y[T:]).all() and not torch.isnan(c.layer.y[:T]).any()


@pytest.mark.parametrize("max_tokens", [40, 300])
def test_counts_of_every_batch(B, max_tokens):
    c = Case(B, max_tokens, 3, 12, 7, count=True)
    total = torch.zeros(12, dtype=torch.int64)
    for i, T in enumerate((1, 40, 7, 64, 65, 300, 2)):
        if T > max_tokens:
            continue
        ids = c.check(T, T <= 64, seed=i)
        n = torch.bincount(ids.reshape(-1), minlength=12)
        total += n
        assert torch.equal(c.layer.counts.cpu().long(), n) and torch.equal(c.layer.cum_counts.cpu().long(), total)


def test_layer_norms_with_biases(B):
    g = torch.Generator().manual_seed(4)
    w = lambda: (1 + 0.1 * torch.randn(256, generator=g)).bfloat16()
    b = lambda: (0.3 * torch.randn(256, generator=g)).bfloat16()
    c = Case(B, 200, 3, 12, 7, kind=B.NORM_LAYER, norm_b=b(), post_w=w(), post_b=b(), next_w=w(), next_b=b())
    for T in (1, 33, 200):
        c.check(T, T <= 64)


@pytest.mark.parametrize("T,n", [(40, 23), (64, 0), (300, 65), (300, 64), (300, 299), (300, 0)])
def test_padding_rows_and_a_gate_per_token(B, T, n):
    """Live rows as the definition has them, the others neither read nor written."""
    w = torch.ones(256).bfloat16()
    c = Case(B, 300, 3, 12, 7, post_w=w, next_w=w, count=True)
    g = torch.Generator().manual_seed(T + n)
    r, gate = torch.randn(T, 256, generator=g), torch.rand(T, 1, generator=g) + 0.5
    ref, ids = c.definition(r)
    rc = r.cuda()
    rc[n:] = float("nan")
    out, x = torch.full((T, 256), -7.0, device="cuda"), torch.full((T, 256), -7.0, dtype=torch.bfloat16, device="cuda")
    c.layer.forward(rc, out, x, gate=gate.cuda(), n_valid=torch.tensor([n], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(c.layer.status.item()) == 0 and (out[n:] == -7).all() and (x[n:] == -7).all()
    assert torch.equal(c.layer.counts.cpu().long(), torch.bincount(ids[:n].reshape(-1), minlength=12))
    if n == 0:
        return
    tol = 5e-3 if T <= 64 else 6e-2
    ref = gate.double() * ref
    upd = out.double().cpu() - r.double()
    assert float((upd[:n] - ref[:n]).norm() / ref[:n].norm()) < tol
    ref = c.norm(r.double() + ref, w, None)
    assert float((x.double().cpu()[:n] - ref[:n]).norm() / ref[:n].norm()) < tol


def test_bf16_experts(B):
    c = Case(B, 200, 3, 12, 7, bf16=True)
    for T in (1, 64, 65, 200):
        c.check(T, True)                                              # no 8-bit activations on either path
