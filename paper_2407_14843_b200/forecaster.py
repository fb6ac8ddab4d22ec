"""Arrival-rate forecaster on the forecasting operators, and the stability test that it feeds.

The paper's optimizer predicts the largest arrival rate of the next seconds with a small recurrent
network (Section "Optimizer") and calls a workload stable when the horizontal solver returns the
same configuration for the current and for the predicted rate (Section "Transition").  Here the
network is a stack of selective state space blocks (``forecast.ssm_scan`` / ``ssm_step`` between two
``forecast.linear``), so that a pipeline's history is read in one pass and every further second
costs one step per pipeline, and the predicted rates stay on the device for the solver.

    python -m paper_2407_14843_b200.forecaster [--pipelines N] [--seconds L] [--steps K] [--ticks T]

trains on synthetic one-second rates, warms the pipelines' states up and then runs ticks: forecast,
two horizontal solves, stability flags.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import forecast

HORIZON = 10        # seconds ahead whose largest rate is predicted
N_FEATURES = 8      # inputs of a second (three used; rows of 16 bytes)
MIN_RATE = 1e-3     # rps; what an idle second counts as, in features, targets and predictions alike


def features(rates: torch.Tensor, first_second: int = 0) -> torch.Tensor:
    """[batch, length] rates (rps) -> [batch, length, N_FEATURES] bfloat16: logarithm, time of day."""
    t = torch.arange(first_second, first_second + rates.shape[1], device=rates.device, dtype=torch.float32)
    phase = (2 * math.pi / 86400) * t
    out = torch.zeros(*rates.shape, N_FEATURES, device=rates.device)
    out[..., 0] = 0.25 * torch.log(rates.float().clamp(min=MIN_RATE))
    out[..., 1] = torch.sin(phase)
    out[..., 2] = torch.cos(phase)
    return out.bfloat16()


class RateForecaster:
    """Predicts, for every second of a pipeline's rates, the logarithm of the largest rate of the next ``HORIZON``
    seconds over the current one.  Parameters are float32; the matrix products take them as bfloat16."""

    def __init__(self, width: int = 64, inner: int = 128, state: int = 16, conv_width: int = 4, layers: int = 2, seed: int = 0,
                 device="cuda"):
        self.inner, self.state, self.conv_width, self.layers = inner, state, conv_width, layers
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)

        def matrix(n, k, gain=1.0):
            return torch.randn(n, k, generator=g) * (gain / math.sqrt(k))

        p = {"embed": matrix(width, N_FEATURES, 2.0), "embed_bias": torch.zeros(width),
             "head": matrix(8, width, 0.1), "head_bias": torch.zeros(8)}
        for i in range(layers):
            step = torch.exp(torch.rand(inner, generator=g) * math.log(100.0)) * 1e-3      # 0.001 .. 0.1
            p.update({
                f"in{i}": matrix(2 * inner + 2 * state, width), f"dt{i}": matrix(inner, width, 0.1),
                f"out{i}": matrix(width, inner, 1 / math.sqrt(2 * layers)), f"out_bias{i}": torch.zeros(width),
                f"a_log{i}": torch.log(torch.arange(1, state + 1).float()).repeat(inner, 1),
                f"conv{i}": matrix(inner, conv_width), f"conv_bias{i}": torch.zeros(inner),
                f"skip{i}": torch.ones(inner), f"dt_bias{i}": step + torch.log(-torch.expm1(-step))})
        self.params = {k: v.to(device).requires_grad_() for k, v in p.items()}
        self.device = torch.device(device)

    def _w(self, name: str) -> torch.Tensor:
        return self.params[name].bfloat16()

    def _block_inputs(self, i: int, h: torch.Tensor):
        """Normalised input's projections: gate, x, B, C, dt."""
        n, s = self.inner, self.state
        u = (h.float() * torch.rsqrt(h.float().square().mean(-1, keepdim=True) + 1e-6)).bfloat16()
        z, x, b, c = forecast.Linear.apply(u, self._w(f"in{i}")).split([n, n, s, s], dim=-1)
        return z, x, b, c, forecast.Linear.apply(u, self._w(f"dt{i}"))

    def _parameters(self, i: int):
        p = self.params
        return (-torch.exp(p[f"a_log{i}"]), p[f"conv{i}"], p[f"conv_bias{i}"], p[f"skip{i}"], p[f"dt_bias{i}"])

    def _head(self, h: torch.Tensor) -> torch.Tensor:
        return forecast.Linear.apply(h, self._w("head"), self.params["head_bias"])[:, 0].float()

    def _scan(self, x: torch.Tensor, lengths: Optional[torch.Tensor], keep_states: bool):
        """[batch, length, features] -> ([batch * length] outputs, states)."""
        rows, length = x.shape[:2]
        h = forecast.Linear.apply(x.reshape(rows * length, -1), self._w("embed"), self.params["embed_bias"])
        states = []
        for i in range(self.layers):
            z, u, b, c, dt = (t.unflatten(0, (rows, length)) for t in self._block_inputs(i, h))
            a, conv, conv_bias, skip, dt_bias = self._parameters(i)
            if keep_states:
                r = forecast.ssm_scan(u, dt, a, b, c, conv, conv_bias, skip, dt_bias, z, lengths=lengths)
                y = r.y
                states.append((r.conv_state, r.ssm_state))
            else:
                y = forecast.SsmScan.apply(u, dt, a, b, c, conv, conv_bias, skip, dt_bias, z, lengths)
            h = forecast.Linear.apply(y.flatten(0, 1), self._w(f"out{i}"), self.params[f"out_bias{i}"], "none", h)
        return self._head(h), states

    def loss(self, rates: torch.Tensor) -> torch.Tensor:
        """Mean squared error of the predicted logarithm over [batch, length + HORIZON] rates."""
        seen = rates[:, :-HORIZON]
        ahead = rates[:, 1:].unfold(1, HORIZON, 1).amax(-1)
        target = torch.log(ahead.clamp(min=MIN_RATE) / seen.clamp(min=MIN_RATE))
        out, _ = self._scan(features(seen), None, False)
        return (out - target.flatten()).square().mean()

    def train_step(self, rates: torch.Tensor, optimizer: torch.optim.Optimizer) -> torch.Tensor:
        optimizer.zero_grad(set_to_none=True)
        loss = self.loss(rates)
        loss.backward()
        optimizer.step()
        return loss.detach()

    @torch.no_grad()
    def warm_up(self, rates: torch.Tensor, lengths: Optional[torch.Tensor] = None):
        """Reads [batch, length] rates (row b only up to ``lengths[b]``); returns the states for ``tick``."""
        return self._scan(features(rates), lengths, True)[1]

    @torch.no_grad()
    def tick(self, states, rates: torch.Tensor, second: int) -> torch.Tensor:
        """One second of every pipeline: updates ``states`` in place and returns the predicted rates (rps)."""
        h = forecast.linear(features(rates[:, None], second)[:, 0], self._w("embed"), self.params["embed_bias"])
        for i, (conv_state, ssm_state) in enumerate(states):
            z, u, b, c, dt = self._block_inputs(i, h)
            a, conv, conv_bias, skip, dt_bias = self._parameters(i)
            y = forecast.ssm_step(u, dt, a, b, c, conv, conv_bias, skip, dt_bias, z, conv_state=conv_state, ssm_state=ssm_state)
            h = forecast.linear(y, self._w(f"out{i}"), self.params[f"out_bias{i}"], residual=h)
        return rates.float().clamp(min=MIN_RATE) * torch.exp(self._head(h))


def to_mrps(rates: torch.Tensor) -> torch.Tensor:
    """Rates (rps) as the solvers take them: whole milli-requests per second, at least 1000."""
    return torch.ceil(rates.double() * 1000).clamp(1000, 4e9).to(torch.int64).to(torch.uint32)


class StabilityMonitor:
    """Horizontal solves at the current and at the predicted rate, and their comparison."""

    def __init__(self, workload):
        from . import solver
        self.solver, self.problem = solver, solver.Problem.of_workload(workload)
        self.dev = solver.workload_to_device(workload)
        self.workspace = solver.alloc_workspace(self.problem, False)
        self.current, self.predicted = (solver.alloc_result(workload.n_instances, workload.n_stages) for _ in range(2))
        self.stable = torch.empty(workload.n_instances, dtype=torch.int32, device="cuda")

    def __call__(self, current: torch.Tensor, predicted: torch.Tensor) -> torch.Tensor:
        for rates, out in ((current, self.current), (predicted, self.predicted)):
            self.solver.themis_solve_horizontal_batch(self.problem, self.dev["lat_us"], self.dev["profile_id"], to_mrps(rates), out,
                                                      self.workspace)
        self.solver.themis_configs_equal_batch(self.current, self.predicted, self.stable)
        return self.stable


def main(argv=None) -> None:
    import argparse

    from . import workloads
    ap = argparse.ArgumentParser(description="Train an arrival-rate forecaster on synthetic rates and run ticks.")
    ap.add_argument("--pipelines", type=int, default=256)
    ap.add_argument("--seconds", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--ticks", type=int, default=20)
    args = ap.parse_args(argv)

    traces = torch.from_numpy(workloads.rate_traces(1, args.pipelines, args.seconds + HORIZON + args.ticks)).cuda()
    model = RateForecaster()
    optimizer = torch.optim.Adam(model.params.values(), lr=3e-3)
    for k in range(args.steps):
        loss = model.train_step(traces[:, :args.seconds + HORIZON], optimizer)
        if k % 10 == 0 or k + 1 == args.steps:
            print(f"step {k}: mean squared error of the logarithm {loss.item():.4f}")

    pipelines = workloads.make_horizontal_workload(args.pipelines)
    monitor = StabilityMonitor(pipelines)
    states = model.warm_up(traces[:, :args.seconds])
    stable = 0
    for t in range(args.seconds, args.seconds + args.ticks):
        predicted = model.tick(states, traces[:, t], t)
        stable += int(monitor(traces[:, t], predicted).sum())
    forecast.check_status()
    print(f"{args.ticks} ticks of {args.pipelines} pipelines: {stable / (args.ticks * args.pipelines):.3f} of the workloads stable")


if __name__ == "__main__":
    main()
