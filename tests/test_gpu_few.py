"""tempo_few_ffn / tempo_few_ffn_bf16 against the layer's definition in 64 bits.

Tolerances (derived): out is rounded to bf16 once, 2^-8 of the value at most.  H enters the down product with 8
significant bits in the fp8 call (two e4m3 terms: at most 2^-8 of the value, plus 2^-17 of its block's largest) and 16 in
the bf16 call; both GEMMs accumulate in 32 bits (2^-16 of the sum of magnitudes is granted for up to 8192 terms).
Element by element that bounds the error by 2^-8 |out| + c S with S = sum_s |w| sum_j |W2_j h_j|, c = 2^-8 + 2^-13 (fp8) or
2^-13 (bf16).  Roundings of random sign add up to far less, so the mean is held too: a bf16 rounding has a relative
root mean square of 1.7e-3, the two-term split of H 0.7e-3: rms(err) / rms(out) <= 2.5e-3 (fp8) and 2.1e-3 (bf16)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


class Layer:
    """Seeded weights of G instance slots, packed on the GPU, and the definition on the CPU in 64 bits."""

    def __init__(self, B, G, d, f, bf16, seed=0):
        self.B, self.G, self.d, self.f, self.bf16 = B, G, d, f, bf16
        g = torch.Generator().manual_seed(seed)
        w13, w2 = torch.randn(G, 2 * f, d, generator=g) * 0.05, torch.randn(G, d, f, generator=g) * 0.05
        self.shape0 = B.make_shape(1, 1, 1, G, 1, d, f, 128)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        if bf16:
            a, b = w13.bfloat16(), w2.bfloat16()
            self.packed = torch.empty(B.tempo_packed_weight_bytes_bf16(self.shape0), dtype=torch.uint8, device="cuda")
            B.tempo_pack_weights_bf16(self.shape0, a.cuda(), b.cuda(), self.packed)
            self.w13, self.w2 = a.double(), b.double()
        else:
            (qa, sa, self.w13), (qb, sb, self.w2) = self._quantise(w13, g), self._quantise(w2, g)
            self.packed = torch.empty(B.tempo_packed_weight_bytes(self.shape0), dtype=torch.uint8, device="cuda")
            B.tempo_pack_weights(self.shape0, qa.cuda(), sa.cuda(), qb.cuda(), sb.cuda(), self.packed, self.status)
        torch.cuda.synchronize()

    @staticmethod
    def _quantise(w, g):
        G, n, k = w.shape
        blk = w.view(G, n // 128, 128, k // 128, 128)
        blk = blk * torch.exp2(torch.randint(-3, 4, (G, n // 128, 1, k // 128, 1), generator=g).float())   # scales that differ
        s = torch.exp2(torch.ceil(torch.log2(blk.abs().amax(dim=(2, 4), keepdim=True) / 448)))
        q = (blk / s).to(torch.float8_e4m3fn)
        return q.view(torch.uint8).reshape(G, n, k), s.reshape(G, n // 128, k // 128).contiguous(), \
            (q.double() * s.double()).reshape(G, n, k)

    def run(self, x, ids, w, rmap, n_valid=None, workspace=None, repeat=1):
        T, k = ids.shape
        E, R = rmap.shape
        shape = self.B.make_shape(T, k, E, self.G, R, self.d, self.f, 128)
        if workspace is None:
            workspace = torch.zeros(self.B.tempo_few_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
        out = torch.full((T + 1, self.d), -77.0, dtype=torch.bfloat16, device="cuda")
        self.status.zero_()
        nv = None if n_valid is None else torch.tensor([n_valid], dtype=torch.int32, device="cuda")
        fn = self.B.tempo_few_ffn_bf16 if self.bf16 else self.B.tempo_few_ffn
        xc, ic, wc, rc = x.cuda(), ids.cuda(), w.cuda(), rmap.cuda()
        for _ in range(repeat):
            fn(shape, xc, ic, wc, nv, rc, self.packed, out[:T], self.status, workspace)
        torch.cuda.synchronize()
        assert (out[T] == -77).all()
        return out[:T].cpu(), int(self.status.item())

    def definition(self, x, ids, w, rmap, n_valid=None):
        T, k = ids.shape
        E, R = rmap.shape
        out, mag = torch.zeros(T, self.d, dtype=torch.float64), torch.zeros(T, self.d, dtype=torch.float64)
        for t in range(T if n_valid is None else n_valid):
            for s in range(k):
                e = int(ids[t, s])
                slots = [int(v) for v in rmap[e]] if 0 <= e < E else []
                slot = next((v for v in slots if 0 <= v < self.G), None)
                if slot is None:
                    continue
                gu = self.w13[slot] @ x[t].double()
                gate, up = gu[:self.f], gu[self.f:]
                h = gate * torch.sigmoid(gate) * up
                out[t] += float(w[t, s]) * (self.w2[slot] @ h)
                mag[t] += abs(float(w[t, s])) * (self.w2[slot].abs() @ h.abs())
        return out, mag

    def check(self, got, ref, mag):
        got = got.double()
        c = 2.0 ** -13 if self.bf16 else 2.0 ** -8 + 2.0 ** -13
        err = (got - ref).abs()
        assert (err <= 2.0 ** -8 * ref.abs() + c * mag + 1e-30).all()
        if ref.numel() >= 1024 and (ref != 0).any():
            rel = float(err.pow(2).mean().sqrt() / ref.pow(2).mean().sqrt())
            assert rel <= (2.1e-3 if self.bf16 else 2.5e-3), rel


def batch(T, k, E, d, seed, distinct=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g).bfloat16()
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]) if distinct else torch.randint(0, E, (T, k), generator=g)
    return x, ids.int(), torch.rand(T, k, generator=g) + 0.05


def plain_map(E, G):
    m = torch.full((E, 1), -1, dtype=torch.int32)
    m[:min(E, G), 0] = torch.arange(min(E, G), dtype=torch.int32)
    return m


CASES = [  # T, k, E, G, d, f
    (1, 1, 1, 1, 128, 128),
    (1, 2, 4, 4, 256, 512),
    (1, 8, 16, 16, 1024, 384),
    (2, 2, 3, 3, 384, 640),
    (5, 2, 8, 8, 256, 512),
    (8, 4, 8, 8, 512, 256),
    (9, 3, 12, 5, 640, 384),              # most experts elsewhere
    (16, 2, 4, 4, 384, 256),
    (17, 8, 40, 33, 128, 128),
    (33, 2, 6, 6, 256, 384),              # one accumulator slot
    (40, 1, 1, 1, 896, 256),              # every token on one expert
    (64, 16, 64, 64, 256, 128),           # 1024 pairs
    (64, 1, 2, 2, 512, 1024),
    (31, 32, 32, 32, 128, 256),
]


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
@pytest.mark.parametrize("T,k,E,G,d,f", CASES)
def test_few_matches_the_definition(B, T, k, E, G, d, f, bf16):
    L = Layer(B, G, d, f, bf16, seed=T + d)
    x, ids, w = batch(T, k, E, d, seed=T * 13 + k)
    m = plain_map(E, G)
    got, st = L.run(x, ids, w, m)
    assert st == 0
    L.check(got, *L.definition(x, ids, w, m))


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
def test_wide_layer_split_over_all_sms(B, bf16):
    L = Layer(B, 3, 4096, 1536, bf16)
    x, ids, w = batch(3, 2, 3, 4096, seed=1)
    m = plain_map(3, 3)
    got, st = L.run(x, ids, w, m)
    assert st == 0
    L.check(got, *L.definition(x, ids, w, m))


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
def test_one_workspace_serves_calls_of_many_sizes(B, bf16):
    """Counters are handed from call to call; fewer tokens than the workspace was sized for; the same bits every time."""
    L = Layer(B, 8, 256, 384, bf16)
    ws = torch.zeros(B.tempo_few_workspace_bytes(B.make_shape(64, 4, 8, 8, 1, 256, 384, 128)), dtype=torch.uint8, device="cuda")
    m = plain_map(8, 8)
    seen = {}
    for i, (T, k) in enumerate([(64, 4), (1, 1), (7, 2), (64, 4), (33, 3), (1, 1), (64, 4), (16, 4), (7, 2)]):
        x, ids, w = batch(T, k, 8, 256, seed=T)
        got, st = L.run(x, ids, w, m, workspace=ws, repeat=1 + i % 3)
        assert st == 0
        if (T, k) in seen:
            assert torch.equal(got, seen[T, k])
        seen[T, k] = got
        L.check(got, *L.definition(x, ids, w, m))


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
@pytest.mark.parametrize("n_valid", [0, 1, 9, 12])
def test_padding_remote_repeated_and_bad_ids(B, bf16, n_valid):
    L = Layer(B, 6, 256, 256, bf16)
    x, ids, w = batch(12, 4, 10, 256, seed=2, distinct=False)      # experts may repeat within a token
    ids[0] = ids[0, 0]
    ids[3] = 9                                                      # a token with no expert here
    ids[5, 1], ids[6, 0], ids[11, 2] = -1, 10, 2 ** 30              # not experts
    m = torch.full((10, 3), -1, dtype=torch.int32)                  # replicas: the first column with a slot counts
    m[:6, 1] = torch.arange(6, dtype=torch.int32)
    m[2, 0], m[2, 2], m[4, 0] = 5, 1, 77                            # 77 is no slot of this rank
    got, st = L.run(x, ids, w, m, n_valid=n_valid)
    bad = any(not 0 <= int(e) < 10 for e in ids[:n_valid].reshape(-1))
    assert st == (B.STATUS_BAD_ID if bad else 0)
    L.check(got, *L.definition(x, ids, w, m, n_valid))
    assert (got[n_valid:] == 0).all()
    if n_valid > 3:
        assert (got[3] == 0).all()


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
def test_values_of_every_size(B, bf16):
    """Tokens whose values differ by many orders of magnitude, within a row and between rows; zeros; a row that is not
    finite makes its own output NaN and no other."""
    L = Layer(B, 4, 512, 256, bf16)
    x, ids, w = batch(10, 2, 4, 512, seed=4)
    m = plain_map(4, 4)
    x = x.float()
    x[1] *= 1e-4
    x[2] *= 30
    x[3, ::7] *= 1e-3
    x[4] = 0
    x[5, 128:256] = 0
    x = x.bfloat16()
    clean, st = L.run(x, ids, w, m)
    ref, mag = L.definition(x, ids, w, m)
    for t in range(10):
        L.check(clean[t:t + 1], ref[t:t + 1], mag[t:t + 1])
    assert (clean[4] == 0).all() and st == 0
    x[6, 5], x[7, 300], x[8, 17] = float("nan"), float("inf"), float("-inf")
    got, _ = L.run(x, ids, w, m)
    assert torch.isnan(got[6:9]).all()
    keep = [0, 1, 2, 3, 4, 5, 9]
    assert torch.equal(got[keep], clean[keep])


def test_graph_stream_and_chain_with_the_router(B):
    """Router and experts captured in a graph on a side stream, replayed with other inputs."""
    L = Layer(B, 16, 512, 256, False)
    T, k, E = 6, 4, 16
    shape = B.make_shape(T, k, E, 16, 1, 512, 256, 128)
    ws = torch.zeros(B.tempo_few_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    wr = (torch.randn(E, 512, generator=torch.Generator().manual_seed(1)) * 0.05).bfloat16()
    m = plain_map(E, 16)
    xc, ids, w = torch.zeros(T, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda"), \
        torch.zeros(T, k, device="cuda")
    out, st = torch.zeros(T, 512, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    wrc, mc = wr.cuda(), m.cuda()

    def layer():
        B.tempo_route(shape, xc, wrc, None, None, ids, w, st)
        B.tempo_few_ffn(shape, xc, ids, w, None, mc, L.packed, out, st, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _ in range(3):
            layer()
    for seed in range(4):
        x, _, _ = batch(T, k, E, 512, seed=seed)
        xc.copy_(x)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        L.check(out.cpu(), *L.definition(x, ids.cpu(), w.cpu(), m))


def test_same_experts_as_the_four_step_block(B):
    """The few-token layer and the four-step block read the same packed weights; they differ by the block's 8-bit
    activations (about 2^-4 of a value each, averaged over the sums)."""
    from paper_2608_13057_b200 import workloads as W
    wl = W.config1()
    buf = B.RankBuffers.for_workload(wl)
    buf.run_block()
    ws = torch.zeros(B.tempo_few_workspace_bytes(buf.shape), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(buf.out)
    B.tempo_few_ffn(buf.shape, buf.x, buf.topk_ids, buf.topk_w, buf.n_valid, buf.replica_map, buf.packed, out, buf.status, ws)
    torch.cuda.synchronize()
    assert int(buf.status.item()) == 0
    a, b = buf.out.double(), out.double()
    assert float((a - b).pow(2).mean().sqrt() / b.pow(2).mean().sqrt()) < 0.06


def test_refusals(B):
    L = Layer(B, 2, 128, 128, False)
    x, ids, w = batch(4, 2, 2, 128, seed=0)
    m = plain_map(2, 2)
    shape = B.make_shape(4, 2, 2, 2, 1, 128, 128, 128)
    ws = torch.zeros(B.tempo_few_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    xc, ic, wc, mc = x.cuda(), ids.cuda(), w.cuda(), m.cuda()
    out = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    st = L.status

    def call(shape=shape, x=xc, ids=ic, w=wc, m=mc, packed=L.packed, out=out, ws=ws):
        B.tempo_few_ffn(shape, x, ids, w, None, m, packed, out, st, ws)

    for kw in (dict(x=x), dict(x=xc.float()), dict(ids=ic.long()), dict(w=None), dict(ws=None), dict(m=None), dict(out=out.t()),
               dict(shape=B.make_shape(65, 2, 2, 2, 1, 128, 128, 128)), dict(shape=B.make_shape(64, 17, 20, 2, 1, 128, 128, 128)),
               dict(shape=B.make_shape(4, 2, 2, 2, 1, 192, 128, 128)), dict(shape=B.make_shape(0, 2, 2, 2, 1, 128, 128, 128)),
               dict(ws=ws[16:]), dict(packed=L.packed[16:]), dict(ws=ws[:-256]), dict(packed=L.packed[:-1024]), dict(x=xc[:3]),
               dict(x=torch.zeros(4 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, 128))):
        with pytest.raises(B.TempoError):
            call(**kw)
    with pytest.raises(B.TempoError):
        B.tempo_few_workspace_bytes(B.make_shape(65, 2, 2, 2, 1, 128, 128, 128))
    call()
    torch.cuda.synchronize()
