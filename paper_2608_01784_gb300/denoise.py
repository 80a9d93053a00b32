"""One denoising forward in 8 bits, from the refinement state to the state of the
next forward:

    counts (reflex_step, ROUTE stage) -> router -> routed experts in 8 bits, with
    the residual, layer by layer -> output head in 8 bits -> sampled tokens and
    their confidences -> commits, history and active blocks (reflex_update_state)

The tokens stay independent of one another between the layers, as in MoEStack; a
layer may have norms in front of and behind its experts, with a gate and a scale on
the way back into the stream (block_norm).
Everything runs in libreflex.so's kernels on the current stream; a forward
allocates nothing and waits for nothing, so it can be captured in a CUDA graph.

    python -m paper_2608_01784_gb300.denoise     a small random model, to the end
"""
from __future__ import annotations

import torch

from . import _binding as B
from . import api


def quantize_layer(w_router: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor,
                   stream=None, norms: dict | None = None) -> dict:
    """A layer of DenoiserFp8: the router [E, d] stays in bf16, the experts go to
    8 bits (quantize_experts).  norms: w_before [d] bf16, by which the layer's normalised
    input is multiplied, and what block_norm takes for its output: w_after, gate (both
    [d]), scale."""
    layer = dict(w_router=w_router, **api.quantize_experts(w_gate_up, w_down, stream))
    return layer if norms is None else dict(layer, norms=norms)


def _a_header_a_layer(op, layers: int) -> list:
    """The operator's workspace for one call a layer, each 256 bytes after the one
    before: a call's error word lies in front of all that later calls write, so every
    layer's can be read at the end."""
    nbytes, device = op.ws_bytes, op.ws.device
    op.ws = None
    ws = torch.empty(nbytes + 256 * (layers - 1), dtype=torch.uint8, device=device)
    ws[:256 * layers].zero_()
    return [ws[256 * i:256 * i + nbytes] for i in range(layers)]


def _check(t: torch.Tensor, shape: tuple, what: str, device=None):
    if not (t.is_cuda and t.dtype == torch.bfloat16 and tuple(t.shape) == shape
            and t.is_contiguous() and t.device == (device or t.device)):
        raise ValueError(f"{what}: a contiguous CUDA tensor {shape} of torch.bfloat16")


def _norms(layers: list, d: int, final_norm) -> list | None:
    """The layers' norms, checked; None where there are none."""
    norms = [w["norms"] for w in layers if w.get("norms") is not None]
    if len(norms) not in (0, len(layers)) or (final_norm is not None and not norms):
        raise ValueError("norms: in every layer or in none")
    dev = layers[0]["w_router"].device
    for n in norms:
        if not set(n) <= {"w_before", "w_after", "gate", "scale"}:
            raise ValueError("norms: w_before, w_after, gate and scale")
        if n.get("w_before") is None:
            raise ValueError("norms: w_before is needed")
        _check(n["w_before"], (d,), "w_before", dev)
        for name in ("w_after", "gate"):
            if n.get(name) is not None:
                _check(n[name], (d,), name, dev)
    if final_norm is not None:
        _check(final_norm, (d,), "final_norm", dev)
    return norms or None


class DenoiserFp8:
    """Layers (quantize_layer) of one shape, without a shared expert, and an
    output head (codes, scales: quantize_fp8 of [vocab, d] in 128 x 128 blocks),
    with buffers for `max_tokens` tokens.  The router's workspace is that of a whole
    bf16 layer (2.4 GB at 32768 tokens, d = 2048, 64 experts of 1024, 12 slots), of
    which a forward uses the scores and the record alone.  With norms (in every layer or
    in none), the stream is multiplied by its norm and final_norm [d] in front of the
    head, if that is given."""

    def __init__(self, layers: list, head: tuple, *, d: int, E: int, inter: int, k_max: int,
                 max_tokens: int, flags: int = B.REFLEX_FLAG_RENORM_TOPK,
                 final_norm: torch.Tensor | None = None, eps: float = 1e-6):
        if not layers:
            raise ValueError("a denoiser needs at least one layer")
        self.norms = _norms(layers, d, final_norm)
        self.final_norm, self.eps = final_norm, eps
        self.layers, self.flags, self.max_tokens = layers, flags, max_tokens
        # the router, its counts and its record; of the experts it runs nothing
        self.router = api.MoELayer(layers[0], dtype="bf16", d=d, E=E, inter=inter, shared_inter=0,
                                   k_max=k_max, max_tokens=max_tokens)
        shape = dict(d=d, E=E, inter=inter, k_max=k_max, max_tokens=max_tokens)
        self.experts = api.ExpertsFp8(layers[0], **shape)
        for w in layers[1:]:
            self.experts.check_weights(w)
        for w in layers:
            _check(w["w_router"], (E, d), "w_router")
        self._ws = list(zip(_a_header_a_layer(self.router, len(layers)),
                            _a_header_a_layer(self.experts, len(layers))))
        self.router.ws, self.experts.ws = self._ws[0]
        self.head = api.LinearFp8(*head, max_rows=max_tokens)
        if self.head.K != d:
            raise ValueError("the head takes another width than the layers give")
        dev = head[0].device
        self._h = [torch.empty((max_tokens, d), dtype=torch.bfloat16, device=dev)
                   for _ in range(2 if self.norms is None else 3)]
        ld = -(-self.head.N // 8) * 8
        self._logits = torch.empty((max_tokens, ld), dtype=torch.bfloat16,
                                   device=dev)[:, :self.head.N]
        self.k = torch.empty(max_tokens, dtype=torch.int32, device=dev)
        self.k_sum = torch.zeros(1, dtype=torch.int64, device=dev)
        self._status = torch.zeros(3, dtype=torch.int32, device=dev)
        self._committed = torch.empty(max_tokens, dtype=torch.int32, device=dev)

    def logits(self, state: dict, params: B.reflex_alloc_params,
               hidden: torch.Tensor) -> torch.Tensor:
        """hidden [T, d] bf16 through the layers and the head, with the counts of
        `state`: a view [T, vocab] that the next forward overwrites."""
        T = int(hidden.shape[0])
        if T > self.max_tokens:
            raise ValueError("more tokens than the buffers were sized for")
        _check(hidden, (T, self.experts.d), "hidden", self.k.device)
        k, route = self.k[:T], self.flags | B.REFLEX_STAGE_ROUTE
        h = hidden
        if self.norms is not None:
            stream, x, y = (t[:T] for t in self._h)
            api.block_norm(hidden, w_before=self.norms[0]["w_before"], eps=self.eps, out=stream,
                           norm=x)
            h = x
        for i, w in enumerate(self.layers):
            out = self._h[i & 1][:T] if self.norms is None else y
            self.router.w = self.experts.w = w
            self.router.ws, self.experts.ws = self._ws[i]
            if i == 0:  # counts and the first router in one call
                self.router.step(state, params, h, out=out, k_out=k, k_sum=self.k_sum,
                                 status=self._status[:1], flags=route)
            else:
                self.router.forward(h, k, out, route)
            ids, alpha = self.router.routing()
            self.experts.forward(h, ids, alpha, k, out, residual=self.norms is None)
            if self.norms is None:
                h = out
                continue
            # back into the stream, and from there to the next layer or the head
            last = i + 1 == len(self.layers)
            after = self.final_norm if last else self.norms[i + 1]["w_before"]
            api.block_norm(stream, y, w_after=self.norms[i].get("w_after"),
                           gate=self.norms[i].get("gate"), scale=self.norms[i].get("scale", 1.0),
                           w_before=after, eps=self.eps, out=stream,
                           norm=None if after is None else x)
            h = stream if after is None else x
        return self.head.forward(h, self._logits[:T])

    def forward(self, state: dict, params: B.reflex_alloc_params, hidden: torch.Tensor,
                u: torch.Tensor, tokens: torch.Tensor, conf: torch.Tensor,
                num_blocks: torch.Tensor, theta_commit: float, *, committed=None, **settings):
        """One forward on device tensors: `state` moves on by one (update_state);
        tokens int32 [T] and conf fp32 [T] receive what every position that was
        masked would take (-1 and 0 elsewhere).  u [T] holds the uniforms, and
        settings are sample()'s temperature, top_k, top_p and min_p.  Returns the
        numbers of commits, in `committed` or in a buffer that the next forward
        overwrites (up to max_tokens sequences)."""
        masked = state["masked"]
        self._status.zero_()
        logits = self.logits(state, params, hidden)
        api.sample(logits, u, masked=masked, tokens=tokens, conf=conf, status=self._status[1:2],
                   **settings)
        sequences = int(state["active_block"].numel())
        if committed is None and sequences <= self.max_tokens:
            committed = self._committed[:sequences]
        return api.update_state(state, conf, num_blocks, theta_commit, committed=committed,
                                status=self._status[2:])

    def status(self) -> int:
        """The first error of the last forward's steps, in any layer (waits)."""
        codes = [B.reflex_read_status(self._status[i:i + 1]) for i in range(3)]
        codes += [B.reflex_moe_status(ws) for pair in self._ws for ws in pair]
        codes.append(self.head.status())
        return next((c for c in codes if c != B.REFLEX_OK), B.REFLEX_OK)


def main(seed: int = 0, most: int | None = None) -> dict:
    """Two sequences of a small random model from all masked to all committed, or as
    far as `most` forwards take them."""
    from . import trajectory, workloads
    cfg = workloads.CONFIGS["tiny_fp32"].with_(dtype="bf16", n_seq=2)
    vocab, layers = 1000, 2
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(*shape):
        return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()
    weights = [quantize_layer(draw(cfg.E, cfg.d), draw(cfg.E, 2 * cfg.inter, cfg.d),
                              draw(cfg.E, cfg.d, cfg.inter)) for _ in range(layers)]
    head = api.quantize_fp8(draw(vocab, cfg.d), 128)
    net = DenoiserFp8(weights, head, d=cfg.d, E=cfg.E, inter=cfg.inter, k_max=cfg.k_max,
                      max_tokens=cfg.T)
    start = trajectory.initial_state(workloads.make_state(cfg, seed))
    blocks = torch.from_numpy(trajectory.num_blocks(start)).cuda()
    state = api.state_to_device(start)
    params = B.make_params(**cfg.alloc_params())
    embed, mask_row = draw(vocab, cfg.d) * 16, draw(1, cfg.d) * 16
    place = draw(cfg.T, cfg.d) * 16
    text = torch.full((cfg.T,), -1, dtype=torch.int32, device="cuda")
    tokens, conf = torch.empty_like(text), torch.empty(cfg.T, device="cuda")
    settings = dict(temperature=torch.full((cfg.T,), 0.8, device="cuda"),
                    top_p=torch.full((cfg.T,), 0.95, device="cuda"))
    forwards = 0
    while forwards != most and bool((state["active_block"] <= blocks).any()):
        known = (text >= 0)[:, None]
        hidden = (torch.where(known, embed[text.clamp(min=0).long()], mask_row) + place)
        before = state["masked"].clone()
        net.forward(state, params, hidden, torch.rand(cfg.T, generator=g, device="cuda"), tokens,
                    conf, blocks, 0.5, **settings)
        text = torch.where((before == 1) & (state["masked"] == 0), tokens, text)
        forwards += 1
    code = net.status()
    if code != B.REFLEX_OK:
        raise B.ReflexError(code, "DenoiserFp8.forward")
    return dict(text=text, forwards=forwards, state=state, vocab=vocab)


if __name__ == "__main__":
    done = main()
    print(f"{int((done['text'] >= 0).sum())} positions in {done['forwards']} forwards")
