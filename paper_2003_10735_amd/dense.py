"""Trainable parts between a frozen front part's features and the head, trained together with the head: a 1x1 layer in 8-bit integers
(DenseFront) and a residual block of two layers in bfloat16 (DenseBlockFront).

The layer maps every cell of the feature map (a token) from the front's channels to the head's.  Its products run in 8-bit integers
(st_int8_linear, st_int8_linear_backward), its gradient comes from the head's full backward pass (st_partial_distill with feature_grad),
and AdamW (st_adamw_step) updates it with states of 8 or 32 bits; the head takes the library's own descent in the same call.
"""
from __future__ import annotations

import math
from dataclasses import replace

import paper_2003_10735_amd as st


class _CountedSteps:
    """A count of the steps that parameters have taken, where whether the last one was taken is on the device: its gradients' norm goes to pinned
    memory behind it and is looked at when the count is asked for next."""

    def _start_counting(self):
        import torch
        self._steps, self._last = 0, None        # _last: recorded behind the last step, while it is not known whether it was taken
        self._last_norm = torch.empty(1, dtype=torch.float32, pin_memory=True)

    @property
    def steps(self) -> int:
        """Steps that the layer has taken.  Waits for the last one, if it may have been left out."""
        if self._last is not None:
            self._last.synchronize()
            self._last = None
            if not math.isfinite(self._last_norm.item()):
                self._steps -= 1
        return self._steps

    @steps.setter
    def steps(self, taken: int):
        self._steps, self._last = taken, None

    def _left_out_unless_finite(self, norm):
        """The step just enqueued is taken only if this norm is finite."""
        import torch
        if not torch.cuda.is_current_stream_capturing():      # (a recorded step's number is fixed)
            self._last_norm.copy_(norm, non_blocking=True)
            self._last = torch.cuda.Event()
            self._last.record()


class DenseFront(_CountedSteps):
    """weight [desc.c_in, c_front] float32 and bias [desc.c_in] float32 are used in place; desc describes the head behind the layer (its
    feature type and layout are chosen here: bfloat16, channels last).

    With max_norm > 0 a step whose gradients' norm is not finite leaves the layer and its state as they were, and is not counted in `steps`;
    the head, which has its own gradients, takes its step all the same.  Whether a step was taken is on the device: `step` asks for it when it
    enqueues the next one's update, behind everything else of that step, so the device has work meanwhile."""

    def __init__(self, desc: st.HeadDesc, weight, bias, lr: float = 1e-3, weight_decay: float = 0.0, max_norm: float = 1.0,
                 state_bits: int = 8):
        import torch
        self.desc = replace(desc, feat_dtype=st.ST_BF16, feat_layout=st.ST_NHWC)
        self.weight, self.bias, self.lr, self.max_norm = weight, bias, lr, max_norm
        self._start_counting()
        c_out, c_front = weight.shape
        d, device = self.desc, weight.device
        cells = d.n * d.h * d.w
        self.grads = [torch.empty_like(weight), torch.empty_like(bias)]
        params = [weight, bias]
        self.tensors = st.AdamWTensors(params, self.grads, weight_decay=[weight_decay, 0.0], **st.new_adamw_state(params, state_bits))
        self.features = torch.empty((d.n, d.h, d.w, c_out), dtype=torch.bfloat16, device=device)
        self.feature_grad = torch.empty((d.n, c_out, d.h, d.w), dtype=torch.float32, device=device)
        self.loss = torch.empty(2, dtype=torch.float32, device=device)
        self.grad_norm = torch.empty(1, dtype=torch.float32, device=device)
        self.workspaces = (st.new_int8_workspace(cells, c_out, c_front, device=device),
                           st.new_int8_workspace(cells, c_out, c_front, backward=True, device=device),
                           st.new_adamw_workspace(self.tensors), st.new_workspace(self.desc, device))
        self.quantized = st.st_int8_quantize(weight)

    def forward(self, cells):
        """cells [n*h*w, c_front], float32 or bfloat16 -> the head's features [n, h, w, c_in] bfloat16."""
        wq, scale = self.quantized
        st.st_int8_linear(cells, wq, scale, bias=self.bias, out=self.features.view(-1, self.weight.shape[0]), workspace=self.workspaces[0])
        return self.features

    def step(self, cells, labels, head_params, head_lr: float):
        """One step of the layer and of the head on one key frame (or batch).  Returns the loss before the step (on the device)."""
        d = self.desc
        features = self.forward(cells)
        st.st_partial_distill(d, features, labels, head_params, 1, head_lr, losses=self.loss, feature_grad=self.feature_grad,
                              workspace=self.workspaces[3])
        # one frame's gradient lies channel by channel: its cells' rows are its columns, and nothing is copied
        g = self.feature_grad
        dy = g[0].view(d.c_in, d.h * d.w).t() if d.n == 1 else g.permute(0, 2, 3, 1).reshape(-1, d.c_in)
        st.st_int8_linear_backward(cells, None, dy, dw=self.grads[0], db=self.grads[1], workspace=self.workspaces[1])
        self.steps += 1
        st.st_adamw_step(self.tensors, self._steps, self.lr, max_norm=self.max_norm, grad_norm=self.grad_norm, workspace=self.workspaces[2])
        if self.max_norm > 0.0:
            self._left_out_unless_finite(self.grad_norm)
        st.st_int8_quantize(self.weight, *self.quantized)
        return self.loss[0]


class DenseBlockFront(_CountedSteps):
    """features = cells + act(cells W1^T + b1) W2^T + b2 for every cell of the feature map: two st_linear, the second with the residual in its
    epilogue.  w1 [hidden, desc.c_in], b1 [hidden], w2 [desc.c_in, hidden], b2 [desc.c_in] are float32 and used in place; the products take
    bfloat16 copies of the matrices, which the optimiser's step writes.  desc describes the head behind the block (its feature type and
    layout are chosen here: bfloat16, channels last).

    backward() adds one key frame's (or batch's) gradients to those that are there; apply() brings their sum over the frames to its mean, clips
    it by the norm over all four tensors (st_grad_clip: the matrices and the biases are two lists of the optimiser, whose states have
    state_bits and 32 bits) and steps.  step() does both.  Where that norm is not finite (in float32) neither list takes its step, whichever of
    them the value is in, and the step is not counted in `steps`."""

    def __init__(self, desc: st.HeadDesc, w1, b1, w2, b2, activation: int = st.ST_ACT_GELU, lr: float = 1e-3, weight_decay: float = 0.0,
                 max_norm: float = 1.0, state_bits: int = 8):
        import torch
        self.desc = replace(desc, feat_dtype=st.ST_BF16, feat_layout=st.ST_NHWC)
        self.params, self.activation, self.lr, self.max_norm = (w1, b1, w2, b2), activation, lr, max_norm
        self.frames = 0                          # of the gradients that are there
        self._start_counting()
        d, device = self.desc, w1.device
        hidden, cells = w1.shape[0], d.n * d.h * d.w
        self.grads = [torch.zeros_like(p) for p in self.params]
        dw1, db1, dw2, db2 = self.grads
        self.copies = [w.to(torch.bfloat16) for w in (w1, w2)]
        self.all_grads = st.GradTensors(self.grads)
        # A list of the optimiser leaves its step out for its own gradients alone.  So each has one value more, which nothing else uses, and that has
        # for its gradient 0 where the norm of all is finite and NaN where it is not.
        self.left_out, (guard, other) = torch.zeros(1, device=device), torch.zeros(2, 1, device=device)
        matrices, vectors = [w1, w2, guard], [b1, b2, other]
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * 2
        self.matrices = st.AdamWTensors(matrices, [dw1, dw2, self.left_out], copies=[*self.copies, guard.to(torch.bfloat16)],
                                        weight_decay=[*decay, 0.0], **st.new_adamw_state(matrices, state_bits))
        self.biases = st.AdamWTensors(vectors, [db1, db2, self.left_out], **st.new_adamw_state(vectors, 32))
        empty = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device=device)      # noqa: E731
        self.features = empty(d.n, d.h, d.w, d.c_in)
        self.feature_grad = empty(d.n, d.c_in, d.h, d.w, dtype=torch.float32)
        self.pre, self.hidden, self.hidden_grad = (empty(cells, hidden) for _ in range(3))
        self.loss, self.grad_norm = empty(2, dtype=torch.float32), empty(1, dtype=torch.float32)
        self.workspace = st.new_workspace(self.desc, device)
        self.norm_workspace = st.new_grad_workspace(self.all_grads)
        self.step_workspaces = [st.new_adamw_workspace(t) for t in (self.matrices, self.biases)]
        self.linear_workspaces = self.cells_lie = None

    def forward(self, cells):
        """cells [n*h*w, desc.c_in] bfloat16 -> the head's features [n, h, w, c_in] bfloat16."""
        w1, w2 = self.copies
        _, b1, _, b2 = self.params
        y = self.features.view(-1, self.desc.c_in)
        lie = cells.stride(), cells.data_ptr() % 16
        if self.cells_lie != lie:       # scratch is for cells that lie as these do
            self.cells_lie = lie
            dy = self._feature_rows()
            self.linear_workspaces = (st.new_linear_workspace(cells, w1), st.new_linear_workspace(self.hidden, w2),
                                      st.new_linear_workspace(self.hidden, w2, dy), st.new_linear_workspace(cells, None, self.hidden_grad, self.activation))
        ws = self.linear_workspaces
        st.st_linear(cells, w1, b1, self.activation, pre=self.pre, out=self.hidden, workspace=ws[0])
        st.st_linear(self.hidden, w2, b2, residual=cells, out=y, workspace=ws[1])
        return self.features

    def _feature_rows(self):
        """The head's gradient of the features, a cell a row.  (One frame's lies channel by channel: its cells' rows are its columns.)"""
        d, g = self.desc, self.feature_grad
        return g[0].view(d.c_in, d.h * d.w).t() if d.n == 1 else g.permute(0, 2, 3, 1).reshape(-1, d.c_in)

    def backward(self, cells, labels, head_params, head_lr: float):
        """Forward pass, the head's step on one key frame (or batch), and the block's gradients, added to those of earlier frames.  Returns
        the loss before the head's step (on the device)."""
        st.st_partial_distill(self.desc, self.forward(cells), labels, head_params, 1, head_lr, losses=self.loss, feature_grad=self.feature_grad,
                              workspace=self.workspace)
        dw1, db1, dw2, db2 = self.grads
        more, ws = self.frames > 0, self.linear_workspaces
        st.st_linear_backward(self.hidden, self.copies[1], self._feature_rows(), dx=self.hidden_grad, dw=dw2, db=db2, accumulate=more, workspace=ws[2])
        st.st_linear_backward(cells, None, self.hidden_grad, self.pre, self.activation, dw=dw1, db=db1, accumulate=more, workspace=ws[3])
        self.frames += 1
        return self.loss[0]

    def apply(self):
        """One step with the mean of the gradients that are there, if its norm is finite."""
        if not self.frames:
            return
        import torch
        st.st_grad_clip(self.all_grads, max_norm=self.max_norm, grad_scale=1.0 / self.frames, grad_norm=self.grad_norm, workspace=self.norm_workspace)
        torch.mul(self.grad_norm, 0.0, out=self.left_out)
        self.frames = 0
        self.steps += 1
        for tensors, ws in zip((self.matrices, self.biases), self.step_workspaces):
            # (a limit that nothing finite reaches: it is asked for what is not)
            st.st_adamw_step(tensors, self._steps, self.lr, max_norm=3e38, workspace=ws)
        self._left_out_unless_finite(self.grad_norm)

    def step(self, cells, labels, head_params, head_lr: float):
        """backward() and apply().  Returns the loss before the step (on the device)."""
        loss = self.backward(cells, labels, head_params, head_lr)
        self.apply()
        return loss
