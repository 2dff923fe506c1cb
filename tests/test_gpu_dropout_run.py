"""Dropout in training runs (agn_options.dropout) against the oracle's event loop with the mask that
agn_dropout's definition gives, and evaluation on 4-bit layers (agn_evaluate_mx4) after it."""

import numpy as np
import pytest

import agn_inputs as I
import ops_ref as R
import oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


class DropoutMLP(O.MLP):
    """The oracle's MLP with inverted dropout after each hidden ReLU.  agn_run calls loss_grad
    lam times for each commit in schedule order: that says whose step it is."""

    def __init__(self, dims, p, seed, lam, worker, n):
        super().__init__(dims)
        self.p, self.seed, self.lam, self.worker = p, seed, lam, worker
        self.calls, self.steps = 0, [0] * n

    def loss_grad(self, theta, X, y):
        w = int(self.worker[self.calls // self.lam])
        t, self.steps[w] = self.steps[w], self.steps[w] + 1
        self.calls += 1
        params, L, m = self.unpack(theta), len(self.dims) - 1, len(X)
        h, gain = [X.astype(self.dtype)], R.gain(self.p)
        for l, (W, b) in enumerate(params):
            z = h[-1] @ W.T + b
            if l + 1 < L:
                d = self.dims[l + 1]
                keep = R.keep_mask(m, d, self.p, R.hidden_seed(self.seed, w, l, L - 1), t * m * -(-d // 4))
                z = np.maximum(z, 0.0) * keep * gain
            h.append(z)
        loss, dz = O.softmax_xent(h[-1], y)
        grad = np.zeros(self.num_params)
        for l in range(L - 1, -1, -1):
            ow, ob, oe = self.offsets[l]
            grad[ow:ob], grad[ob:oe] = (dz.T @ h[l]).ravel(), dz.sum(axis=0)
            if l > 0:
                dz = (dz @ params[l][0]) * (h[l] > 0) * gain
        return loss, grad


def run(agn, dims, m, n, lam, C, seed, p, eta=0.05, split_calls=False, **kw):
    N = n * 3 * m
    w, t = I.make_schedule(n, C + n, 0, 2, seed)
    ds = I.SyntheticDataset(seed, dims[0], N, I.DIST_UNIFORM, (dims[0], 64, dims[-1]), N // n)
    okw = {}
    if kw.get("elide_accumulator"):
        okw["elide_accumulator"] = True
    if kw.get("local_optimizer") == agn.AGN_OPT_ADAM:
        okw["optimizer"] = "adam"
    ref = O.agn_run(DropoutMLP(dims, p, seed, lam, w, n), I.init_params(seed, dims), n, lam, eta, w[:C], t[:C],
                    ds, m, N // n, **okw)
    with agn.AGN(dims, n, lam, eta, seed, batch=m, n_samples=N, dropout=p, **kw) as h:
        if split_calls:
            h.run(C // 2, w, t)
            h.run(C - C // 2, w[C // 2:], t[C // 2:])
        else:
            h.run(C, w, t)
        return h.central().astype(np.float64), h.loss(), ref


def rel(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


# fp32 runs without dropout are held to 1e-5 of the oracle after these few commits; the mask adds two
# roundings of 2^-24 a layer to them
@pytest.mark.parametrize("dims,m,kw", [
    ((64, 48, 32, 10), 16, {}),                                     # tensor cores, three bf16 pieces
    ((64, 48, 32, 10), 16, dict(gemm=1)),                           # CUDA cores
    ((70, 33, 21, 10), 20, {}),                                     # odd widths
    ((64, 40, 10), 33, {}),                                         # one hidden layer
    ((96, 64, 64, 40), 40, {}),                                     # a wide output layer
    ((64, 64, 64, 64, 10), 16, dict(tc_mask=2 | 4)),                # forward on the CUDA cores
    ((64, 64, 64, 64, 10), 16, dict(tc_mask=1 | 4)),                # dX there
    ((64, 64, 64, 64, 10), 16, dict(tc_mask=64)),                   # gathered minibatches
    ((64, 48, 32, 10), 16, dict(elide_accumulator=1)),
    ((256, 136, 200, 10), 130, {}),                                 # several column tiles, split K
], ids=str)
def test_fp32_runs(agn, dims, m, kw):
    got, loss, ref = run(agn, dims, m, 4, 3, 9, 17, 0.4, **kw)
    assert rel(got, ref.theta) < 1e-5
    np.testing.assert_allclose(loss, ref.loss, rtol=1e-5, atol=1e-5)


def test_adam(agn):
    """Adam divides by the root of the second moment: 1e-4, as its runs without dropout."""
    got, loss, ref = run(agn, (64, 48, 32, 10), 16, 3, 3, 7, 11, 0.25, eta=1e-3,
                         local_optimizer=agn.AGN_OPT_ADAM)
    assert rel(got, ref.theta) < 1e-4
    np.testing.assert_allclose(loss, ref.loss, rtol=1e-4, atol=1e-4)


def test_steps_continue_over_calls(agn):
    got, _, ref = run(agn, (64, 48, 32, 10), 16, 3, 2, 8, 5, 0.5, split_calls=True)
    assert rel(got, ref.theta) < 1e-5


@pytest.mark.parametrize("gemm", [0, 1])
def test_bf16_runs(agn, gemm):
    """bf16's criterion: each commit's loss within 2e-2 of the oracle's."""
    _, loss, ref = run(agn, (128, 128, 64, 10), 32, 4, 3, 9, 23, 0.3, precision=agn.AGN_PREC_BF16, gemm=gemm)
    assert np.max(np.abs(loss - ref.loss)) < 2e-2


def test_bf16_kept_steps(agn):
    """Waves whose steps' activations are kept (dropped ones among them): the same criterion."""
    _, loss, ref = run(agn, (256, 2048, 2048, 10), 32, 8, 4, 8, 3, 0.3, eta=0.01, precision=agn.AGN_PREC_BF16)
    assert np.max(np.abs(loss - ref.loss)) < 2e-2


@pytest.mark.parametrize("kw", [{}, dict(precision=1), dict(gemm=1)], ids=str)
def test_no_dropout_is_the_run_without_the_option(agn, kw):
    dims, n, lam, seed = (64, 48, 32, 10), 3, 3, 7
    out = []
    for p in (None, 0.0):
        with agn.AGN(dims, n, lam, 0.1, seed, batch=16, n_samples=192, **kw, **({} if p is None else {"dropout": p})) as h:
            h.run(9)
            out.append(h.central())
    assert np.array_equal(out[0], out[1])


@pytest.mark.parametrize("p", [1.0, -0.5, float("nan")])
def test_refuses(agn, p):
    with pytest.raises(agn.AGNError) as e:
        agn.AGN((64, 48, 10), 2, 1, 0.1, 1, dropout=p)
    assert e.value.code == agn.AGN_E_INVALID and "dropout" in str(e.value)


# ------------------------------------------------------------ 4-bit evaluation

def evaluated_by_definition(dims, theta, X, y):
    """Loss and logits with the hidden layers in 4 bits, sums in 64 bits, values that the library has in
    fp32 rounded to it."""
    offs, h = O.MLP(dims).unpack(np.asarray(theta, np.float64)), X.astype(np.float64)
    for l, (W, b) in enumerate(offs):
        if l + 1 == len(offs):
            z = h @ W.T + b
            break
        q = R.mx4_values(*R.mx4_quantize(h))[:, :h.shape[1]]
        wq = R.mx4_values(*R.mx4_quantize(W))[:, :W.shape[1]]
        h = np.maximum(q @ wq.T + b, 0).astype(np.float32).astype(np.float64)
    loss, _ = O.softmax_xent(z, y)
    return loss, z


@pytest.mark.parametrize("dims,E,kw", [((64, 48, 32, 10), 300, {}), ((70, 33, 10), 129, {}), ((64, 40, 36, 50), 200, {}),
                                       ((64, 352, 352, 10), 9000, {}), ((96, 30, 20, 10), 5000, dict(gemm=1))], ids=str)
def test_evaluate_mx4(agn, dims, E, kw):
    n, m, seed, N = 3, 16, 31, 144
    with agn.AGN(dims, n, 2, 0.05, seed, batch=m, n_samples=N, n_eval=E, eval_mx4=1, dropout=0.2, **kw) as h:
        plain = h.evaluate()
        h.run(6)
        for _ in range(2):   # theta~ as it is at the call
            loss, acc, pred = h.evaluate_mx4(with_pred=True)
            theta = h.central()
            rows = N + np.arange(E)
            X = I.make_inputs_x(seed, dims[0], rows, I.DIST_UNIFORM)
            y = I.teacher_labels(X, I.teacher_params(seed, (dims[0], 64, dims[-1])), I.DIST_UNIFORM)
            want, z = evaluated_by_definition(dims, theta, X, y)
            # a hidden sum that fp32 rounds at a border of the codes moves a few samples' logits: 1e-4 of the loss
            assert abs(loss - want) < 1e-4 * want
            top = np.sort(z, 1)
            clear = top[:, -1] - top[:, -2] > 1e-3 * np.abs(z).max()
            assert np.mean(pred[clear] != np.argmax(z[clear], 1)) < 2e-3
            assert abs(acc - np.mean(pred == y)) < 1e-6
            h.run(3)
        # the two evaluations do not disturb each other
        a = h.evaluate()
        h.evaluate_mx4()
        assert h.evaluate() == a and a != plain


def test_evaluate_mx4_is_the_operators_by_hand(agn):
    """Train with dropout, then the same layers through the public calls."""
    import torch
    dims, E, n, seed, N = (784, 200, 72, 10), 400, 4, 5, 256
    with agn.AGN(dims, n, 3, 0.05, seed, batch=32, n_samples=N, n_eval=E, eval_mx4=1, dropout=0.5) as h:
        h.run(8)
        theta = h.central()
        _, _, pred = h.evaluate_mx4(with_pred=True)
    x = torch.tensor(I.make_inputs_x(seed, dims[0], N + np.arange(E), I.DIST_UNIFORM), device="cuda")

    def matrix(r, c):
        return tuple(torch.empty(b, dtype=torch.uint8, device="cuda") for b in agn.agn_mx4_bytes(r, c))
    q = matrix(E, dims[0])
    agn.agn_mx4_quantize(x, 0, E, dims[0], *q)
    params = [(torch.tensor(W, device="cuda"), torch.tensor(b, device="cuda")) for W, b in O.MLP(dims).unpack(theta)]
    for l, (W, b) in enumerate(params[:-1]):
        wq, last = matrix(dims[l + 1], dims[l]), l == len(params) - 2
        agn.agn_mx4_quantize(W, 0, dims[l + 1], dims[l], *wq)
        out = (torch.empty(E, dims[l + 1], device="cuda"), None) if last else matrix(E, dims[l + 1])
        agn.agn_mx4_linear(*q, *wq, E, dims[l], dims[l + 1], out[0], 0 if last else agn.AGN_PREC_MX4, bias=b, relu=1,
                           y_scales=out[1])
        q = out
    z = q[0].double() @ params[-1][0].double().T + params[-1][1].double()
    top = z.sort(1)[0]
    clear = (top[:, -1] - top[:, -2] > 1e-5 * z.abs().max()).cpu().numpy()   # fp32 sums of 72 terms: 72 2^-24
    assert clear.mean() > 0.95 and np.array_equal(z.argmax(1).cpu().numpy()[clear], pred[clear])


def test_evaluate_mx4_refusals(agn):
    with pytest.raises(agn.AGNError) as e:
        agn.AGN((64, 48, 10), 2, 1, 0.1, 1, eval_mx4=1)
    assert e.value.code == agn.AGN_E_INVALID
    with pytest.raises(agn.AGNError) as e:
        agn.AGN((64, 10), 2, 1, 0.1, 1, n_eval=10, eval_mx4=1)
    assert e.value.code == agn.AGN_E_UNSUPPORTED
    with agn.AGN((64, 48, 10), 2, 1, 0.1, 1, n_eval=10) as h:
        with pytest.raises(agn.AGNError) as e:
            h.evaluate_mx4()
        assert e.value.code == agn.AGN_E_INVALID
    with agn.AGN((64, 48, 10), 2, 1, 0.1, 1, n_eval=10, eval_mx4=1) as h:
        with pytest.raises(agn.AGNError) as e:
            agn.agn_evaluate_mx4(h.h, np.empty(9, np.int32))
        assert e.value.code == agn.AGN_E_INVALID
