"""The operators round the grouped products as they are used together: a mixture of networks with a norm in front and dropout behind, eagerly, on
other streams and in a captured graph; dropout in the trainer; rows far apart.  Needs an MI355X."""
import math

import numpy as np
import pytest
import torch

import routed_reference as ref
import train_reference as train_ref
from paper_2212_01185_amd import binding, synth, train
from train_reference import assert_near

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
ROWS, WIDTH, HIDDEN, EXPERTS, CHOICES, DROP, SEED = 700, 160, 128, 6, 2, 0.2, 77


def _parameters(seed):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return {"gamma": (1 + 0.2 * normal(1, WIDTH)).cuda(), "beta": (0.2 * normal(1, WIDTH)).cuda(),
            "gate": (2 * normal(1, EXPERTS, WIDTH) / math.sqrt(WIDTH)).to(BF16).cuda(),
            "w1": (normal(EXPERTS, HIDDEN, WIDTH) * math.sqrt(2 / WIDTH)).to(BF16).cuda(), "b1": (0.1 * normal(EXPERTS, HIDDEN)).cuda(),
            "w2": (normal(EXPERTS, WIDTH, HIDDEN) / math.sqrt(HIDDEN)).to(BF16).cuda(), "b2": (0.1 * normal(EXPERTS, WIDTH)).cuda()}


def _layer(x, g, p, step, all_rows):
    """The layer's result and, for the gradient g of it, the gradients of x and of all parameters; the choices."""
    xn, stats = binding.pcc_layer_norm(x, p["gamma"], p["beta"], out_dtype=BF16)
    logits = binding.pcc_grouped_linear(xn, p["gate"], None, all_rows)
    expert, weight = binding.pcc_route(logits, CHOICES)
    offsets, place = binding.pcc_expert_sort(expert, EXPERTS)
    rows = binding.pcc_expert_rows(xn, place)
    h = binding.pcc_grouped_linear(rows, p["w1"], p["b1"], offsets, binding.PCC_ACT_RELU)
    z = binding.pcc_grouped_linear(h, p["w2"], p["b2"], offsets)
    y = binding.pcc_expert_join(z, place, weight, out_dtype=FP32)
    out = binding.pcc_dropout(y, DROP, SEED, step=step, residual=x)

    dy = binding.pcc_dropout(g, DROP, SEED, step=step)
    dz, dweight = binding.pcc_expert_join_grad(dy, z, place, weight)
    dh, dw2, db2 = binding.pcc_grouped_linear_grad(dz, h, p["w2"], offsets, binding.PCC_ACT_RELU)
    drows, dw1, db1 = binding.pcc_grouped_linear_grad(dh, rows, p["w1"], offsets)
    dlogits = binding.pcc_route_grad(dweight, logits, expert, weight)
    dxn, dgate, _ = binding.pcc_grouped_linear_grad(dlogits, xn, p["gate"], all_rows)
    dxn = binding.pcc_expert_join(drows, place, out_dtype=FP32) + dxn
    dx, dgamma, dbeta = binding.pcc_layer_norm_grad(dxn, x, stats, p["gamma"])
    return {"out": out, "x": g + dx, "gamma": dgamma, "beta": dbeta, "gate": dgate, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2}, expert


class _Round(torch.autograd.Function):
    """Rounding to bf16 of the value, of its gradient, or of both."""

    @staticmethod
    def forward(ctx, x, there, back):
        ctx.back = back
        return x.to(BF16).double() if there else x.clone()

    @staticmethod
    def backward(ctx, g):
        return (g.to(BF16).double() if ctx.back else g), None, None


def _reference(x, g, p, step, expert):
    """The same in 64 bits on the CPU by automatic differentiation, with the given choices, rounded where the operators round."""
    x = x.double().cpu().requires_grad_(True)
    p = {k: v.double().cpu().requires_grad_(True) for k, v in p.items()}
    h = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, keepdim=True, correction=0) + 1e-5)
    xn = _Round.apply(p["gamma"] * h + p["beta"], True, False)
    logits = _Round.apply(_Round.apply(xn, False, True) @ p["gate"][0].T, True, True)
    weight = torch.softmax(torch.gather(logits, 1, expert), 1)
    y = torch.zeros_like(x)
    for e in range(EXPERTS):
        token, slot = torch.nonzero(expert == e, as_tuple=True)
        rows = _Round.apply(xn[token], False, True)
        hidden = _Round.apply(torch.relu(_Round.apply(rows @ p["w1"][e].T + p["b1"][e], False, True)), True, False)
        z = _Round.apply(hidden @ p["w2"][e].T + p["b2"][e], True, True)
        y = y.index_add(0, token, z * weight[token, slot][:, None])
    border = round(DROP * 65536)
    kept = (ref.drop_bits(range(len(x)), WIDTH, SEED, step) >= border).double()
    out = x + y * kept / (1 - border / 65536)
    (out * g.double().cpu()).sum().backward()
    return dict({k: v.grad for k, v in p.items()}, x=x.grad, out=out.detach())


def _inputs(seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(ROWS, WIDTH, generator=gen).cuda(), torch.randn(ROWS, WIDTH, generator=gen).cuda()


def test_a_mixture_forward_and_backward():
    x, g = _inputs(1)
    p = _parameters(2)
    got, expert = _layer(x, g, p, torch.tensor([3]).cuda(), torch.tensor([0, ROWS]).cuda())
    want = _reference(x, g, p, 3, expert.long().cpu())
    # Values next to a border of bf16 may be rounded to the other side, since sums are in fp32: off by 2^-20 of their size after some 200
    # products where a step is 2^-8, one in 2^11; with the cancellation of a sum of random signs (14 times smaller than the sum of sizes) one in
    # 150.  Each such value is off by 2^-8, as independent errors 2^-8 / sqrt(150) = 3.2e-4 of a layer's norm; nine roundings lie on
    # the longest way: 1e-3.  4e-3 leaves a factor of four.
    for name, value in want.items():
        off = (got[name].double().cpu().view(value.shape) - value).norm() / value.norm()
        assert off <= 4e-3, (name, off.item())


def test_a_mixture_on_another_stream_and_captured():
    """Replays see new inputs, another mask each time by the step's number, and other choices; each gives the eager call's bits."""
    p, all_rows = _parameters(5), torch.tensor([0, ROWS]).cuda()
    x, g = _inputs(6)
    step = torch.tensor([10]).cuda()
    want, _ = _layer(x, g, p, step, all_rows)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = _layer(x, g, p, step, all_rows)
    side.synchronize()
    assert all(torch.equal(want[k], got[k]) for k in want)
    source, gradient = x.clone(), g.clone()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    captured = []
    torch.cuda.synchronize()
    for graph in graphs:
        with torch.cuda.graph(graph):
            captured.append(_layer(source, gradient, p, step, all_rows)[0])
    for k in range(4):
        now = _inputs(20 + k)
        source.copy_(now[0])
        gradient.copy_(now[1])
        step.fill_(100 + k)
        eager = {name: t.clone() for name, t in _layer(now[0], now[1], p, step, all_rows)[0].items()}
        torch.cuda.synchronize()
        for graph, result in zip(graphs, captured):
            graph.replay()
        torch.cuda.synchronize()
        for result in captured:
            assert all(torch.equal(eager[name], result[name]) for name in eager), k


def test_many_calls_at_once_on_streams():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(40000, 160, generator=gen).to(BF16).cuda()
    gamma = torch.ones(2, 160, device="cuda")
    off = torch.tensor([0, 15000, 40000]).cuda()
    expert = torch.randint(0, 30, (40000, 2), generator=gen, dtype=torch.int32).cuda()

    def calls():
        y, stats = binding.pcc_layer_norm(x, gamma, None, off)
        return (y,) + tuple(binding.pcc_layer_norm_grad(y, x, stats, gamma, off)) + tuple(binding.pcc_expert_sort(expert, 30))

    want = calls()
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                results.append(calls())
    torch.cuda.synchronize()
    for got in results:
        assert all(torch.equal(a, b) for a, b in zip(want, got))


# ---------------------------------------------------------------------------------------------------- rows and elements behind the 2^32nd

FAR = 1 << 22


def _far(rows, width, dtype, fill):
    """A matrix whose rows are 2^22 elements apart; only its own elements are set."""
    full = torch.empty(rows * FAR, dtype=dtype, device="cuda")
    t = full.view(rows, FAR)[:, :width]
    t.copy_(fill) if isinstance(fill, torch.Tensor) else t.fill_(fill)
    return t


def test_rows_far_apart():
    rows, width = 1030, 40                          # the last rows lie behind the 2^32nd element
    gen = torch.Generator().manual_seed(2)
    values, residual = torch.randn(rows, width, generator=gen).to(BF16), torch.randn(rows, width, generator=gen).to(BF16)
    x, out = _far(rows, width, BF16, values.cuda()), _far(rows, width, BF16, 5.0)
    near = values.cuda()
    y, stats = binding.pcc_layer_norm(near)
    y2, stats2 = binding.pcc_layer_norm(x, out=out)
    assert torch.equal(y, y2) and torch.equal(stats, stats2)
    for a, b in zip(binding.pcc_layer_norm_grad(near, near, stats), binding.pcc_layer_norm_grad(x, x, stats, dx=out)):
        assert torch.equal(a, b)
    assert torch.equal(binding.pcc_dropout(near, 0.3, 1, residual=residual.cuda()), binding.pcc_dropout(x, 0.3, 1, residual=residual.cuda(), out=out))
    place = torch.randperm(rows, generator=gen).to(torch.int32).view(rows, 1).cuda()
    weight = torch.rand(rows, 1, generator=gen).cuda()
    assert torch.equal(binding.pcc_expert_rows(near, place), binding.pcc_expert_rows(x, place, out=out))
    assert torch.equal(binding.pcc_expert_join(near, place, weight), binding.pcc_expert_join(x, place, weight, out=out))
    for a, b in zip(binding.pcc_expert_join_grad(near, near, place, weight), binding.pcc_expert_join_grad(x, x, place, weight, dz=out)):
        assert torch.equal(a, b)
    expert, w = binding.pcc_route(near, 3, over_all=True)
    for a, b in zip((expert, w), binding.pcc_route(x, 3, over_all=True)):
        assert torch.equal(a, b)
    assert torch.equal(binding.pcc_route_grad(w, near, expert, w, over_all=True), binding.pcc_route_grad(w, x, expert, w, over_all=True, dlogits=out))


def test_more_than_2_to_the_32_elements():
    """Rows one behind the other whose last elements have numbers beyond 32 bits."""
    rows, width = (1 << 32) // 4096 + 100, 4096
    x = torch.zeros(rows, width, dtype=BF16, device="cuda")
    gen = torch.Generator().manual_seed(3)
    x[-50:] = torch.randn(50, width, generator=gen).to(BF16).cuda()
    y, stats = binding.pcc_layer_norm(x)
    (want, bound), _ = ref.layer_norm(x[-50:], None, None, [0, 50], 1e-5)
    assert_near(y[-50:], want, bound, "y")
    dx, dgamma, dbeta = binding.pcc_layer_norm_grad(x, x, stats, dx=y)
    for got, (value, limit) in zip((dx[-50:], dgamma, dbeta), ref.layer_norm_grad(x[-50:], x[-50:], stats[-50:], None, [0, 50])):
        # (the sums are over all rows: zeros but for the last)
        assert_near(got, value, limit * 4, "gradient")
    out = binding.pcc_dropout(x, 0.25, 9, out=y)
    wanted, limit = ref.dropout(x[-2:], 0.25, None, ref.drop_bits(range(rows - 2, rows), width, 9, 0))
    assert_near(out[-2:], wanted, limit, "dropout")


# ---------------------------------------------------------------------------------------------------- as many groups as there may be, any address

@pytest.mark.parametrize("groups,features", [(65535, 24), (65535, 9), (3000, 200)])
def test_layer_norm_of_as_many_groups_as_there_may_be(groups, features):
    gen = torch.Generator().manual_seed(groups)
    lengths = torch.randint(0, 3, (groups,), generator=gen)
    lengths[[0, 64, 65, groups - 2]] = torch.tensor([900, 0, 1500, 700])
    off = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)])
    rows = int(off[-1])
    x, dy = torch.randn(rows, features, generator=gen), torch.randn(rows, features, generator=gen)
    gamma, beta = torch.randn(groups, features, generator=gen), torch.randn(groups, features, generator=gen)
    g = torch.repeat_interleave(torch.arange(groups), lengths)
    y, stats = binding.pcc_layer_norm(x.cuda(), gamma.cuda(), beta.cuda(), off.cuda())
    dx, dgamma, dbeta = binding.pcc_layer_norm_grad(dy.cuda(), x.cuda(), stats, gamma.cuda(), off.cuda())
    # one group of all rows with each row's own weights: h and the sums of a row do not hang on the group
    (h, e_h), _ = ref.layer_norm(x, None, None, [0, rows], 1e-5)
    want = gamma.double()[g] * h + beta.double()[g]
    assert_near(y, want, gamma.double()[g].abs() * e_h + 2 * ref.U * (want.abs() + (gamma.double()[g] * h).abs()), "y")
    (value, limit), _, _ = ref.layer_norm_grad(dy.double() * gamma.double()[g], x, stats, None, [0, rows])
    assert_near(dx, value, limit * (1 + 2 * ref.U), "dx")       # (the product with gamma is rounded in the kernel: in the reference's bound of u)
    s = stats.double().cpu()
    part = dy.double() * ((x.double() - s[:, :1]) * s[:, 1:])
    for name, got, p in (("dgamma", dgamma, part), ("dbeta", dbeta, dy.double())):
        sums, sizes = (torch.zeros(groups, features, dtype=torch.float64).index_add_(0, g, t) for t in (p, p.abs()))
        assert_near(got, sums, (lengths[:, None].double() + 8) * ref.U * sizes, name)
        assert (got.cpu()[lengths == 0] == 0).all()


def _shifted(t):
    """The same values one element behind the start of an allocation."""
    full = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    full[1:] = t.reshape(-1)
    return full[1:].view(t.shape)


@pytest.mark.parametrize("features", [40, 37, 4100])
def test_weights_statistics_and_places_at_any_address(features):
    gen = torch.Generator().manual_seed(features)
    x, dy = torch.randn(2100, features, generator=gen).to(BF16).cuda(), torch.randn(2100, features, generator=gen).to(BF16).cuda()
    gamma, beta, off = torch.randn(2, features, generator=gen).cuda(), torch.randn(2, features, generator=gen).cuda(), torch.tensor([0, 1999, 2100]).cuda()
    y, stats = binding.pcc_layer_norm(x, gamma, beta, off)
    y2, stats2 = binding.pcc_layer_norm(_shifted(x), _shifted(gamma), _shifted(beta), off, out=_shifted(torch.zeros_like(x)), stats=_shifted(torch.zeros_like(stats)))
    assert torch.equal(y, y2) and torch.equal(stats, stats2)
    want = binding.pcc_layer_norm_grad(dy, x, stats, gamma, off)
    got = binding.pcc_layer_norm_grad(_shifted(dy), _shifted(x), _shifted(stats), _shifted(gamma), off, dx=_shifted(torch.zeros_like(x)),
                                      dgamma=_shifted(torch.zeros_like(gamma)), dbeta=_shifted(torch.zeros_like(gamma)))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    logits, dweight = torch.randn(300, 21, generator=gen).cuda(), torch.randn(300, 3, generator=gen).cuda()
    expert, weight = binding.pcc_route(logits, 3)
    again = binding.pcc_route(_shifted(logits), 3, expert=_shifted(torch.zeros_like(expert)), weight=_shifted(torch.zeros_like(weight)))
    assert torch.equal(expert, again[0]) and torch.equal(weight, again[1])
    assert torch.equal(binding.pcc_route_grad(dweight, logits, expert, weight),
                       binding.pcc_route_grad(_shifted(dweight), _shifted(logits), _shifted(expert), _shifted(weight), dlogits=_shifted(torch.zeros_like(logits))))
    offsets, place = binding.pcc_expert_sort(expert, 21)
    again = binding.pcc_expert_sort(_shifted(expert), 21, offsets=_shifted(torch.zeros_like(offsets)), place=_shifted(torch.zeros_like(place)))
    assert torch.equal(offsets, again[0]) and torch.equal(place, again[1])
    rows = binding.pcc_expert_rows(x[:300], place)
    assert torch.equal(rows, binding.pcc_expert_rows(_shifted(x[:300]), _shifted(place), out=_shifted(torch.zeros_like(rows))))
    assert torch.equal(binding.pcc_expert_join(rows, place, weight),
                       binding.pcc_expert_join(_shifted(rows), _shifted(place), _shifted(weight), out=_shifted(torch.zeros(300, features, dtype=BF16, device="cuda"))))
    want = binding.pcc_expert_join_grad(dy[:300], rows, place, weight)
    got = binding.pcc_expert_join_grad(_shifted(dy[:300]), _shifted(rows), _shifted(place), _shifted(weight), dz=_shifted(torch.zeros_like(rows)),
                                       dweight=_shifted(torch.zeros_like(weight)))
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_types_that_no_operator_has_are_refused():
    x, place = torch.zeros(4, 8, dtype=BF16, device="cuda"), torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    for bad in (lambda: binding.pcc_layer_norm(x, out_dtype=torch.float64), lambda: binding.pcc_layer_norm(x, out_dtype=FP16), lambda: binding.pcc_layer_norm(x, out_dtype=FP32),
                lambda: binding.pcc_dropout(x, 0.1, 1, out_dtype=FP16), lambda: binding.pcc_dropout(x, 0.1, 1, out_dtype=torch.float64),
                lambda: binding.pcc_expert_join(x, place, out_dtype=FP16), lambda: binding.pcc_route(x, 9), lambda: binding.pcc_route(x, 0), lambda: binding.pcc_dropout(x, 1.5, 1)):
        with pytest.raises(binding.PccError):
            bad()
    for bad in (lambda: binding.pcc_layer_norm(x.double()), lambda: binding.pcc_layer_norm(x.t()), lambda: binding.pcc_layer_norm(x[:1].expand(4, 8)),
                lambda: binding.pcc_layer_norm(x, torch.ones(2, 8, device="cuda")), lambda: binding.pcc_layer_norm(x, torch.ones(1, 8)),
                lambda: binding.pcc_expert_sort(place, 0), lambda: binding.pcc_expert_sort(place, 1025), lambda: binding.pcc_expert_sort(place.long(), 4),
                lambda: binding.pcc_expert_rows(x[:3], place), lambda: binding.pcc_dropout(x, 0.1, -1), lambda: binding.pcc_dropout(x, 0.1, 1 << 64),
                lambda: binding.pcc_dropout(x, 0.1, 1, residual=x.float())):
        with pytest.raises(ValueError):
            bad()


# ---------------------------------------------------------------------------------------------------- dropout in the trainer

def _picture(h, w):
    return synth.make_image(5, synth.ImageSpec(w, h, 4, 3.0, 12.0))[None]


@pytest.mark.parametrize("name", ["workload", "paper"])
def test_gradients_with_dropout(name):
    blob = (synth.make_blob if name == "workload" else synth.make_paper_blob)(3)
    img = _picture(17, 21)
    trainer = train.Trainer(blob, dropout=0.25, seed=11)
    trainer.optimizer.step.fill_(4)
    bits = trainer.gradients(torch.from_numpy(img).cuda())
    layers, k, nbhd, delay, act, dist = train.parse_blob(blob)
    bf16 = lambda t: t.to(BF16).double()  # noqa: E731
    scale = 1 / (1 - 0.25)
    h, masks = [torch.from_numpy(train_ref.contexts(img, nbhd, delay))], []
    for i, (w, b) in enumerate(layers):
        z = h[-1] @ torch.from_numpy(w.astype(np.float64)).T + torch.from_numpy(b.astype(np.float64))
        if i + 1 < len(layers):
            masks.append((ref.drop_bits(range(len(z)), z.shape[1], 11 + i, 4) >= 16384).double() * scale)
            z = bf16(bf16(train_ref.activate(z, act)) * masks[-1])
        h.append(z)
    rgb = torch.from_numpy(img.reshape(-1, 3))
    want_bits = train_ref.code_length(h[-1], rgb, k, dist).mean().item() / 3
    dz = bf16(train_ref.loss_gradient(h[-1], rgb, k, dist, 1.0 / len(rgb))[0])
    # as without dropout (2e-3: values next to a border of bf16 that fall to its other side), with a second rounding at each layer
    near = 3e-3
    assert abs(bits.item() - want_bits) <= near * want_bits
    for i in reversed(range(len(layers))):
        dw, db = dz.T @ h[i], dz.sum(0)
        got = trainer.dw[i][0].double().cpu()[:, :dw.shape[1]]
        assert (got - dw).norm() <= near * dw.norm() and (trainer.db[i][0].double().cpu() - db).norm() <= near * db.norm(), i
        if i:
            dz = bf16(bf16((dz @ torch.from_numpy(layers[i][0].astype(np.float64))) * train_ref.derivative(h[i], act)) * masks[i - 1])
    assert trainer.blob() == blob


def test_trainer_without_dropout_is_as_it_was_and_masks_change_with_the_step():
    img = torch.from_numpy(_picture(16, 16)).cuda()
    plain, zero = train.Trainer(synth.make_blob(1)), train.Trainer(synth.make_blob(1), dropout=0.0, seed=5)
    assert torch.equal(plain.step(img), zero.step(img)) and all(torch.equal(a, b) for a, b in zip(plain.w, zero.w))
    dropped = train.Trainer(synth.make_blob(1), dropout=0.5, lr=0.0)
    first, again = dropped.gradients(img), dropped.gradients(img)
    dropped.step(img)
    then = dropped.gradients(img)
    assert torch.equal(first, again) and not torch.equal(first, then)
    for bad in (1.0, -0.1, float("nan")):
        with pytest.raises(ValueError):
            train.Trainer(synth.make_blob(1), dropout=bad)


def test_the_command_with_dropout(tmp_path):
    np.save(tmp_path / "p.npy", np.concatenate([_picture(24, 24)] * 2))
    train.main([str(tmp_path / "p.npy"), "--out", str(tmp_path / "m.blob"), "--steps", "2", "--batch", "2", "--crop", "16", "--dropout", "0.1"])
    binding.Codec((tmp_path / "m.blob").read_bytes(), 0).close()
