"""A mixture whose samples are routed to its components (paper_2004_06231_amd/mixture.py): the same results, bit for bit where
the same kernels run on the same rows, as the components' own calls on the samples that the float64 oracle assigns to them."""
import json
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2004_06231_amd as P
import workloads
from oracle import routing as R
from oracle.einet import BERNOULLI, GAUSSIAN
from tests.common import make_oracle
from tests.gpu_common import gpu_model, dev, assert_logp_close

pytestmark = pytest.mark.gpu

SPEC = dict(kind="rat", D=24, depth=3, R=2)
EM = dict(min_var=1e-4, max_var=1.0, w_floor=1e-9)


def components(n, max_batch, family=GAUSSIAN, K=6, seed=41, spec=SPEC):
    oracles, models = [], []
    for c in range(n):
        oracle, flat, _ = make_oracle(spec, K, 1, family, seed + c, leaf_range=(0.2, 0.8))
        oracles.append(oracle)
        models.append(gpu_model(spec, K, 1, family, max_batch, seed + c, flat))
    return oracles, models


def data(N, seed=5):
    rng = np.random.default_rng(seed)
    return workloads.draw_data(rng, dict(kind="gaussian_mixture", components=4, std=0.3), N, 24, 1)


def masks(rng, N, kind):
    if kind == "none":
        return None
    return (rng.random(24 if kind == "shared" else (N, 24)) < 0.7).astype(np.uint8)


@pytest.mark.parametrize("kind", ["none", "shared", "per_sample"])
@pytest.mark.parametrize("streams", [0, 3])
def test_density_and_route_match_oracle(kind, streams):
    oracles, models = components(5, 40)
    x = data(130)
    mask = masks(np.random.default_rng(1), 130, kind)
    coef = np.log(np.array([0.1, 0.3, 0.2, 0.25, 0.15])).astype(np.float32)
    mix = P.Mixture(models, coef, [torch.cuda.Stream() for _ in range(streams)])
    ref = np.stack([o.logp(x, mask) for o in oracles])
    rid, rw, rlogp, _ = R.route(ref, coef, 3, True)
    assert_logp_close(mix.logp(dev(x), dev(mask)), rlogp)
    ids, w, logp = mix.route(dev(x), dev(mask), top=3)
    assert_logp_close(logp, rlogp)
    # log-densities are 1e-4 of their size off: components that are closer than that may change places
    t = ref + coef[:, None]
    close = np.abs(np.diff(np.sort(t, 0)[::-1][:4], axis=0)).min(0) > 3e-4 * np.abs(t).max()
    assert close.sum() > 60
    assert np.array_equal(ids.cpu().numpy()[close], rid[close])
    np.testing.assert_allclose(w.cpu().numpy()[close], rw[close], rtol=0, atol=4e-4 * np.abs(t).max())
    for m in models:
        m.close()


@pytest.mark.parametrize("kind", ["none", "per_sample"])
@pytest.mark.parametrize("streams", [0, 2])
@pytest.mark.parametrize("how", ["best", "draw", "given"])
def test_epoch_is_the_components_own_on_their_samples(kind, streams, how):
    N, M = 210, 4
    _, models = components(M, 32)
    _, alone = components(M, 32)
    x = dev(data(N))
    mask = dev(masks(np.random.default_rng(2), N, kind))
    coef = torch.tensor([0.4, 0.1, 0.3, 0.2], device="cuda").log()
    mix = P.Mixture(models, coef, [torch.cuda.Stream() for _ in range(streams)])
    for epoch in range(2):
        rows = torch.stack([torch.cat([m.logp(x[b:b + 32], mask[b:b + 32] if mask is not None else None) for b in range(0, N, 32)]) for m in alone])
        t = rows.double().cpu().numpy() + coef.double().cpu().numpy()[:, None]
        u = torch.rand(N, generator=torch.Generator(device="cuda").manual_seed(epoch), device="cuda")
        if how == "draw":
            want = np.array([R.choose((rows + coef[:, None])[:, n].double().cpu().numpy(), float(u[n]))[0] for n in range(N)])
        elif how == "given":
            want = np.random.default_rng(epoch).integers(-1, M - 1, N)     # the last component gets none, some samples neither
        else:
            want = t.argmax(0)
        ids, logp = mix.em_epoch(x, mask, batch=16, step=0.5, u=u if how == "draw" else None,
                                 ids=dev(want.astype(np.int32)) if how == "given" else None, **EM)
        assert np.array_equal(ids.cpu().numpy(), want)
        ref = torch.zeros(N, device="cuda")
        for c, m in enumerate(alone):
            mine = torch.as_tensor(np.flatnonzero(want == c)).cuda()
            if len(mine) == 0:
                continue
            lp = torch.empty(len(mine), device="cuda")
            m.em_epoch(x[mine].contiguous(), None if mask is None else mask[mine].contiguous(), batch=16, step=0.5, logp=lp, **EM)
            ref[mine] = lp
        assert torch.equal(logp, ref)
        for a, b in zip(models, alone):
            assert torch.equal(a.params, b.params)
        p = np.exp(t - t.max(0))
        share = (p / p.sum(0)).mean(1)
        new = 0.5 * np.exp(coef.double().cpu().numpy()) + 0.5 * share
        np.testing.assert_allclose(mix.log_coef.double().exp().cpu().numpy(), new, rtol=1e-5)
        coef = mix.log_coef.clone()
    for m in models + alone:
        m.close()


@pytest.mark.parametrize("top", [1, 3])
@pytest.mark.parametrize("kind", ["shared", "per_sample"])
def test_inpainting_is_the_weighted_sum_of_the_components_own(top, kind):
    N, M = 75, 4
    _, models = components(M, 64)
    x = dev(data(N))
    mask = dev(masks(np.random.default_rng(3), N, kind))
    mix = P.Mixture(models)
    u = torch.rand(mix.choices(), N * top, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    got = mix.inpaint(x, mask, u, top=top)
    ids, w, _ = mix.route(x, mask, top)
    first, place = R.sort(ids.cpu().numpy(), M)
    want = np.zeros((N, 24, 1))
    for n in range(N):
        for s in range(top):
            c, at = int(ids[n, s]), int(place[n, s])
            one = models[c].sample(1, u[:, at:at + 1].contiguous(), None, x[n:n + 1], mask[n:n + 1] if mask.dim() == 2 else mask)
            want[n] += float(w[n, s]) * one[0].double().cpu().numpy()
    seen = (mask if mask.dim() == 2 else mask[None].expand(N, 24)).bool().cpu().numpy()
    g = got.cpu().numpy()
    assert np.array_equal(g[seen], x.cpu().numpy()[seen])
    # float32 sums of at most three leaf means below 2
    np.testing.assert_allclose(g, want, rtol=0, atol=4 * 2.0 ** -24 * 2 * top)
    for m in models:
        m.close()


def test_samples_come_from_the_components_drawn():
    N, M = 150, 3
    _, models = components(M, 32, BERNOULLI)
    mix = P.Mixture(models, np.log([0.6, 0.1, 0.3]))
    g = torch.Generator(device="cuda").manual_seed(4)
    uc, u, noise = torch.rand(N, generator=g, device="cuda"), torch.rand(mix.choices(), N, generator=g, device="cuda"), torch.rand(N, 24, 1, generator=g, device="cuda")
    got = mix.sample(uc, u, noise)
    ids = np.array([R.choose(mix.log_coef.double().cpu().numpy(), float(v))[0] for v in uc])
    _, place = R.sort(ids[:, None], M)
    for n in range(N):
        at = int(place[n, 0])
        one = models[ids[n]].sample(1, u[:, at:at + 1].contiguous(), noise[at:at + 1].contiguous())
        assert torch.equal(got[n], one[0])
    # a small temperature leaves the most likely component alone
    ids = P.einet_choose(mix.log_coef[None].expand(N, -1), uc, temperature=0.01)[0]
    assert not bool(ids.any())
    assert mix.sample(uc, u, noise, temperature=0.01).shape == (N, 24, 1)
    for m in models:
        m.close()


def test_training_command_reassigns_samples():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for how in ("best", "draw"):
        r = subprocess.run([sys.executable, "-m", "paper_2004_06231_amd.train", "--components", "2", "--n", "600", "--epochs", "3", "--streams", "2",
                            "--reassign", how], capture_output=True, text=True, timeout=110, cwd=root)
        assert r.returncode == 0, r.stderr[-2000:]
        out = json.loads(r.stdout.strip().splitlines()[-1])
        assert out["reassign"] == how and len(out["samples_moved_per_epoch"]) == 2 and math.isfinite(out["held_out_mixture_mean_logp"])
    r = subprocess.run([sys.executable, "-m", "paper_2004_06231_amd.train", "--graphs", "--reassign", "best"], capture_output=True, text=True,
                       timeout=110, cwd=root)
    assert r.returncode != 0 and "--reassign" in r.stderr


@pytest.mark.parametrize("size", [0.0, -2.0 ** 20, 2.0 ** 20])
def test_components_are_drawn_with_their_coefficients_whatever_the_size_of_the_densities(size):
    """Densities that are equal leave the draw to the coefficients: 0.52 and 0.48, whose logarithms next to 2^20 would be rounded
    to eighths (0.53 and 0.47).  Samples that no component, or one, has a finite density for too."""
    _, models = components(2, 32)

    class Given(P.Mixture):
        def component_logp(self, x, mask=None):
            return rows

    x = dev(data(6))
    rows = torch.full((2, 6), size, device="cuda")
    rows[:, 3] = -math.inf
    rows[0, 4] = -math.inf
    rows[1, 5] = math.inf
    u = torch.tensor([0.515, 0.525, 0.0, 0.5, 0.0, 0.0], device="cuda")
    mix = Given(models, torch.tensor([0.52, 0.48]).log())
    ids, _ = mix.em_epoch(x, batch=16, u=u, **EM)
    assert ids.tolist() == [0, 1, 0, -1, 1, 1]
    for m in models:
        m.close()


def test_components_are_drawn_with_their_coefficients_next_to_closed_ones_and_without_a_number():
    """A component that takes no part (its coefficient -inf, or its density NaN) has no say in how the others are drawn, however much
    larger its density is."""
    _, models = components(3, 32)

    class Given(P.Mixture):
        def component_logp(self, x, mask=None):
            return rows

    x = dev(data(8))
    u = torch.tensor([0.515, 0.525, 0.515, 0.525, 0.0, 0.99, 0.3, 0.3], device="cuda")
    for size in (-2.0 ** 20, 2.0 ** 20):
        rows = torch.full((3, 8), size, device="cuda")
        rows[2] = size + 2.0 ** 21
        rows[2, 2:4] = math.nan
        rows[2, 4] = math.inf                        # (closed: +inf and -inf make no number)
        rows[0, 4:6] = math.nan
        rows[:, 6] = math.nan
        rows[:2, 7] = -math.inf
        mix = Given(models, torch.tensor([0.52, 0.48, 0.0]).log())
        ids, _ = mix.em_epoch(x, batch=16, u=u, **EM)
        assert ids.tolist() == [0, 1, 0, 1, 1, 1, -1, -1]
    for m in models:
        m.close()


def test_training_command_with_a_component_that_keeps_no_samples(monkeypatch, capsys):
    """All samples go to the second component: the line stays valid JSON, the first component's mean is null."""
    from paper_2004_06231_amd import train
    epoch = P.Mixture.em_epoch

    def to_the_second(self, x, mask=None, **args):
        return epoch(self, x, mask, **dict(args, u=None, ids=torch.ones(x.shape[0], dtype=torch.int32, device="cuda")))

    monkeypatch.setattr(P.Mixture, "em_epoch", to_the_second)
    monkeypatch.setattr(sys, "argv", "train --components 2 --n 600 --epochs 2 --streams 2 --reassign best".split())
    train.main()
    line = capsys.readouterr().out.strip().splitlines()[-1]

    def refuse(name):
        raise AssertionError(f"{name} in {line}")

    out = json.loads(line, parse_constant=refuse)
    history = out["train_mean_logp_per_epoch_component0"]
    assert math.isfinite(history[0]) and history[1] is None and math.isfinite(out["held_out_mixture_mean_logp"])


def test_a_model_that_is_several_components_works_on_one_stream():
    """The calls on one model share its workspace: side by side on two streams they would overwrite each other's activations."""
    _, (a, b) = components(2, 32)
    _, (a2, b2) = components(2, 32)
    streams = [torch.cuda.Stream() for _ in range(3)]
    x = dev(data(150))
    mix, plain = P.Mixture([a, b, a, b, a], streams=streams), P.Mixture([a2, b2, a2, b2, a2])
    with mix._beside_each_other() as at:
        used = []
        for c in range(5):
            with at(c):
                used.append(torch.cuda.current_stream())
    assert used == [streams[0], streams[1], streams[0], streams[1], streams[0]]
    assert torch.equal(mix.component_logp(x), plain.component_logp(x))
    ids = torch.arange(150, dtype=torch.int32, device="cuda") % 5
    got, want = mix.em_epoch(x, batch=16, ids=ids, **EM)[1], plain.em_epoch(x, batch=16, ids=ids, **EM)[1]
    assert torch.equal(got, want) and torch.equal(a.params, a2.params) and torch.equal(b.params, b2.params)
    assert torch.equal(mix.log_coef, plain.log_coef)
    for m in (a, b, a2, b2):
        m.close()


def test_inpainting_without_a_component_leaves_zeros():
    _, models = components(2, 32)

    class Given(P.Mixture):
        def component_logp(self, x, mask=None):
            return rows

    x, mask = dev(data(5)), dev(masks(np.random.default_rng(4), 5, "per_sample"))
    rows = torch.zeros(2, 5, device="cuda")
    rows[:, 3] = -math.inf
    mix = Given(models)
    got = mix.inpaint(x, mask, torch.rand(mix.choices(), 10, device="cuda"), top=2)
    seen = mask.bool()[:, :, None]
    assert torch.equal(got[seen], x[seen]) and not bool(got[3][~seen[3]].any()) and bool(got[2][~seen[2]].any())
    for m in models:
        m.close()
