"""A training step of a small tied model through the library: tiled table -> embedding -> two LayerNorms with a residual -> head loss ->
gradients -> tile -> clipped AdamW, against automatic differentiation in 64 bits, and captured and replayed."""
import pytest
import torch

from paper_2407_12075_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, V, D, K = 200, 96, 64, 4


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


class Model:
    def __init__(self, bits):
        self.W = rand(1, V * D) * 0.3
        self.gain = [1 + 0.1 * rand(2 + i, D) for i in range(2)]
        self.offset = [0.1 * rand(4 + i, D) for i in range(2)]
        self.params = [self.W, *self.gain, *self.offset]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.opt = B.tbn_adamw_tensors(self.params, self.grads, *B.tbn_adamw_state(self.params, bits), weight_decay=[0.1, 0, 0, 0, 0])
        self.ids = torch.randint(0, V, (T,), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV)
        self.ids[::17] = -1
        self.targets = self.ids.roll(-1)
        self.n = int(((self.targets >= 0)).sum())
        self.step, self.lr = torch.zeros(1, dtype=torch.int64, device=DEV), torch.full((1,), 1e-3, device=DEV)
        self.dloss = torch.full((T,), 1.0 / self.n, device=DEV)

    def gradients(self):
        head, tile, alpha = B.tbn_tile_fwd(self.W, K, B.ALPHA_PER_TILE)
        head = head.view(V, D)
        e = B.tbn_embedding_tiled_fwd(self.ids, V, D, tile, K, alpha, B.ALPHA_PER_TILE, scale=D ** 0.5, y_dtype=B.F32)
        y1, s1, mean1, rstd1 = B.tbn_layernorm_train_fwd(e, self.gain[0], self.offset[0])
        y2, s2, mean2, rstd2 = B.tbn_layernorm_train_fwd(y1, self.gain[1], self.offset[1], residual=e)
        loss, lse = B.tbn_linear_xent_fwd(y2, head, self.targets)
        dy2, G, _ = B.tbn_linear_xent_bwd(y2, head, self.targets, lse, self.dloss)
        ds2, dg2, db2 = B.tbn_layernorm_bwd(dy2, s2, mean2, rstd2, self.gain[1])
        de, dg1, db1 = B.tbn_layernorm_bwd(ds2, s1, mean1, rstd1, self.gain[0], dsum=ds2)
        B.tbn_embedding_bwd(self.ids, de, V, scale=D ** 0.5, add_to=G)
        dW, _, _ = B.tbn_tile_bwd(G.view(-1), tile, alpha, self.W, K, B.ALPHA_PER_TILE)
        for g, got in zip(self.grads, (dW, dg1, dg2, db1, db2)):
            g.copy_(got)
        return loss

    def update(self, step, lr):
        _, scale = B.tbn_grad_norm(self.opt, 1.0)
        B.tbn_adamw_step(self.opt, step, lr, 0.9, 0.95, 1e-8, grad_scale=scale, seed=5)


def reference(model):
    """The same gradients by automatic differentiation in 64 bits; sign() passes its gradient on, as the tiling module does."""
    W = model.W.double().requires_grad_()
    gain, offset = ([p.double().requires_grad_() for p in ps] for ps in (model.gain, model.offset))
    tiles = W.view(K, -1)
    bits = torch.where(tiles.sum(0) > 0, 1.0, -1.0).double()
    alpha = tiles.abs().mean(1, keepdim=True)
    # value alpha * bits; gradient of alpha through bits as they are, and alpha * G straight to W
    head = (alpha * bits + alpha.detach() * (tiles - tiles.detach())).view(V, D)
    ok = (model.ids >= 0)[:, None]
    e = torch.where(ok, head[model.ids.clamp(min=0)] * D ** 0.5, 0.0)

    def norm(x, g, b):
        var, mu = torch.var_mean(x, 1, correction=0, keepdim=True)
        return (x - mu) / torch.sqrt(var + 1e-5) * g + b
    y = norm(norm(e, gain[0], offset[0]) + e, gain[1], offset[1])
    kept = model.targets >= 0
    loss = torch.nn.functional.cross_entropy((y @ head.t())[kept], model.targets[kept], reduction="none")
    (loss.sum() / model.n).backward()
    return loss, kept, [W.grad.view(-1), gain[0].grad, gain[1].grad, offset[0].grad, offset[1].grad]


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_of_a_step(bits):
    model = Model(bits)
    loss = model.gradients()
    want, kept, grads = reference(model)
    # fp32 throughout; ids that are left out give rows of zeros, whose first norm has h = 0 and rstd = 316 (eps alone), so gradients
    # there grow by 316 twice.  5e-5 of the gradient's size leaves room for some 800 roundings of the largest element.
    assert torch.allclose(loss[kept].double(), want, rtol=1e-5, atol=1e-5)
    for got, ref in zip(model.grads, grads):
        assert (got.double() - ref).norm() <= 5e-5 * ref.norm()


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_equal_eager_ones(bits):
    a, b = Model(bits), Model(bits)
    for m in (a, b):                                                    # first calls outside a capture
        m.gradients()
    for m in (a, b):
        for p, q in zip(m.params, Model(bits).params):
            p.copy_(q)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.loss = b.gradients()
        b.update(b.step, b.lr)
    for t in range(1, 5):
        loss = a.gradients()
        a.update(t, a.lr.item())
        b.step.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, b.loss)
        assert all(torch.equal(p, q) for p, q in zip(a.params, b.params))


def test_two_captured_steps_share_nothing():
    """Two models' graphs replayed on two streams at once."""
    models = [Model(8), Model(32)]
    want = []
    for m in models:
        for t in range(1, 4):
            m.gradients()
            m.update(t, 1e-3)
        want.append([p.clone() for p in m.params])
    models, graphs, streams = [Model(8), Model(32)], [], [torch.cuda.Stream() for _ in range(2)]
    for m, s in zip(models, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            m.step += 1
            m.gradients()
            m.update(m.step, 1e-3)
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for m, w in zip(models, want):
        assert all(torch.equal(p, q) for p, q in zip(m.params, w))
