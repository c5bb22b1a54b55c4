"""The few-token experts where the weights are many: the two-half schedule of the active experts, more than 128 instance slots,
one accumulator slot with several parts of lines per CTA.  Definition in 64 bits on the GPU, tolerances as in test_gpu_few."""
import pytest
import torch

from tests.test_gpu_few import Layer, batch, plain_map

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2608_13057_b200 import binding
    return binding


class LargeLayer(Layer):
    def definition(self, x, ids, w, rmap, n_valid=None):
        T = ids.shape[0] if n_valid is None else n_valid
        out = torch.zeros(ids.shape[0], self.d, dtype=torch.float64, device="cuda")
        mag = torch.zeros_like(out)
        xd = x.cuda().double()
        slot = rmap[:, 0][ids.long()]                               # one replica column, every id an expert
        for e in range(self.G):
            t, j = torch.nonzero(slot[:T] == e, as_tuple=True)
            if t.numel() == 0:
                continue
            wt = w[t, j].double().cuda()[:, None]
            t = t.cuda()
            gate, up = (xd[t] @ self.w13[e].cuda().t()).chunk(2, dim=1)
            h, w2 = gate * torch.sigmoid(gate) * up, self.w2[e].cuda()
            out.index_add_(0, t, h @ w2.t() * wt)
            mag.index_add_(0, t, h.abs() @ w2.abs().t() * wt.abs())
        return out.cpu(), mag.cpu()

    def halves(self, ids):
        """Whether the active experts are taken in two halves: eight gate/up blocks or more per SM in each."""
        A = int((ids.unique() < self.G).sum())
        blocks = A * (self.f // 128) * (self.d // (64 if self.bf16 else 128))
        return A >= 2 and blocks >= 16 * torch.cuda.get_device_properties(0).multi_processor_count


def covering(T, k, E, d, seed):
    """A batch whose T * k pairs go round the experts, so that the first min(T * k, E) of them are active."""
    x, _, w = batch(T, k, E, d, seed)
    return x, (torch.arange(T * k).view(T, k) % E).int(), w


CASES = [  # T, k, E, G, d, f, in two halves (fp8, bf16)
    (1, 8, 8, 8, 4096, 1536, (True, True)),
    (9, 3, 9, 9, 4096, 1536, (True, True)),               # an odd number of experts
    (64, 8, 9, 9, 4096, 1536, (True, True)),              # one accumulator slot
    (5, 1, 5, 5, 4096, 1536, (False, True)),              # below the threshold, above it
    (33, 2, 66, 48, 1024, 1024, (True, True)),            # some experts elsewhere
    (64, 16, 300, 300, 512, 512, (True, True)),           # more than 128 slots
    (11, 6, 256, 200, 512, 384, (False, False)),
    (64, 4, 1024, 700, 128, 128, (False, False)),
]


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
@pytest.mark.parametrize("T,k,E,G,d,f,halves", CASES)
def test_large_layers_match_the_definition(B, T, k, E, G, d, f, halves, bf16):
    L = LargeLayer(B, G, d, f, bf16, seed=T + d)
    x, ids, w = covering(T, k, E, d, seed=T * 13 + k)
    m = plain_map(E, G)
    assert L.halves(ids) == halves[bf16]
    ws = torch.zeros(B.tempo_few_workspace_bytes(B.make_shape(T, k, E, G, 1, d, f, 128)), dtype=torch.uint8, device="cuda")
    got, st = L.run(x, ids, w, m, workspace=ws)
    assert st == 0
    ref, mag = L.definition(x, ids, w, m)
    L.check(got, ref, mag)
    for n in (1, 2):                                                # the counters go from call to call, the bits stay
        again, st = L.run(x, ids, w, m, workspace=ws, repeat=n)
        assert st == 0 and torch.equal(again, got)
    nv = (T + 1) // 2                                               # fewer active experts on the same workspace
    got, st = L.run(x, ids, w, m, n_valid=nv, workspace=ws)
    assert st == 0 and (got[nv:] == 0).all()
    L.check(got, *L.definition(x, ids, w, m, nv))


@pytest.mark.parametrize("bf16", [False, True], ids=["fp8", "bf16"])
def test_random_choices_over_two_halves(B, bf16):
    """Experts with unequal numbers of tokens on both sides of the middle, repeated experts in a token, one workspace."""
    L = LargeLayer(B, 40, 1024, 1024, bf16, seed=1)
    m = plain_map(50, 40)
    ws = torch.zeros(B.tempo_few_workspace_bytes(B.make_shape(64, 8, 50, 40, 1, 1024, 1024, 128)), dtype=torch.uint8, device="cuda")
    for seed, (T, k) in enumerate([(64, 8), (7, 8), (64, 1), (20, 5), (48, 8)]):
        x, ids, w = batch(T, k, 50, 1024, seed=seed, distinct=seed % 2 == 0)
        if seed == 2:
            ids[:50] = 3                                            # most tokens on one expert
        got, st = L.run(x, ids, w, m, workspace=ws)
        assert st == 0
        L.check(got, *L.definition(x, ids, w, m))
