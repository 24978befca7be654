"""Shape groups of a Deflated Muon step (Appendix D, "Grouping": matrices of one shape are stacked into one batch and
the batched range finder runs once per group per optimizer step).

Host-side bookkeeping only, no arithmetic. The library takes wide matrices as they are stored
(polar(M^T) = polar(M)^T is applied logically inside the kernels), so a group is keyed by the STORED shape and
nothing is transposed or copied per step: parameters, momenta and gradients of a group live in one [b, m, n]
buffer each, and the model's own tensors are views into it.
"""
from collections import OrderedDict


def shape_groups(shapes):
    """Indices of the 2-D shapes in `shapes`, grouped by shape in order of first appearance:
    OrderedDict {(m, n): [index, ...]}. Anything that is not two-dimensional is left out."""
    groups = OrderedDict()
    for i, s in enumerate(shapes):
        s = tuple(int(x) for x in s)
        if len(s) != 2:
            continue
        groups.setdefault(s, []).append(i)
    return groups


def stack_group(tensors, indices):
    """One contiguous [b, m, n] buffer holding tensors[i] for i in indices (copied once), and the list of views
    into it, in the same order; assigning the views back to the owners makes later steps copy-free."""
    import torch
    first = tensors[indices[0]]
    buf = torch.empty((len(indices),) + tuple(first.shape), dtype=first.dtype, device=first.device)
    views = []
    for j, i in enumerate(indices):
        t = tensors[i]
        if tuple(t.shape) != tuple(first.shape) or t.dtype != first.dtype or t.device != first.device:
            raise ValueError("tensor %d does not belong to this group" % i)
        buf[j].copy_(t)
        views.append(buf[j])
    return buf, views


def deflation_active(step, total_steps, cutoff=1.0):
    """The deflation cutoff of Section 4 ("Deflation cutoff"): deflation runs during the first `cutoff` fraction of
    the `total_steps` optimizer steps (step counted from 0) and the plain filter after it; cutoff = 1 keeps it on
    throughout, cutoff = 0 is plain Muon."""
    if not 0.0 <= cutoff <= 1.0:
        raise ValueError("cutoff is a fraction of the optimizer steps")
    if step < 0 or total_steps <= 0:
        raise ValueError("step >= 0 and total_steps > 0")
    return step < cutoff * total_steps


def _look_ahead_has_gradients(weights, grads, nesterov):
    """The Nesterov look-ahead is formed with the gradient: a group without one is refused before anything has been changed."""
    if nesterov:
        for shape in weights:
            if grads.get(shape) is None:
                raise ValueError("group %s has no gradient, which nesterov=True needs" % (shape,))


def muon_step_groups(ctx, weights, momenta, grads, lr, mu, window, oversample, power_iters, coeff_schedule,
                     step=None, total_steps=None, cutoff=1.0, **kw):
    """One Deflated Muon step over stacked groups: weights/momenta/grads are dicts {(m, n): [b, m, n] tensor} (grads
    may hold None, unless kw says nesterov=True). `window` is the number k of leading triplets, or a ratio w in (0, 1) meaning k = ceil(w min(m, n));
    `oversample` likewise a count or a ratio delta (Section 3: r = ceil(w m), r' = r + ceil(delta m)). With `step` and
    `total_steps` the deflation cutoff applies: past it the step runs with k = 0, which is the plain Muon step (no
    range finder, no deflation pass, the same filter)."""
    import math
    if step is not None and total_steps is not None and not deflation_active(step, total_steps, cutoff):
        window = 0
    _look_ahead_has_gradients(weights, grads, kw.get("nesterov"))
    for shape, W in weights.items():
        ms = min(shape)
        k = int(math.ceil(window * ms)) if 0 < window < 1 else int(window)
        p = int(math.ceil(oversample * ms)) if 0 < oversample < 1 else int(oversample)
        ctx.defl_muon_step_batched(W, momenta[shape], grads.get(shape), lr, mu, k, p, power_iters, coeff_schedule, **kw)


def optimizer_step_groups(ctx, weights, momenta, grads, lr, mu, window, oversample, power_iters, coeff_schedule, rest, rest_grads, rest_lr,
                          rest_step, max_norm=0.0, adamw=None, **kw):
    """One optimizer step over a whole model: Muon on the stacked matrix groups (as muon_step_groups; kw goes there) and AdamW
    on the rest, a binding.AdamWGroup with one gradient per tensor (None: left alone). The global norm is taken over all
    gradients together; with max_norm > 0 its factor scales both kinds. rest_step is an int64 CUDA tensor [1], the number of
    AdamW steps taken so far: it is advanced on the device. A norm that is not finite leaves the rest and the counter as they are,
    and the matrices take a step along their momentum without the gradient: the factor is on the device, the launches of a Muon step do
    not depend on it, and its momentum rule has a meaning for a gradient of zero. (Who wants such a step left out altogether reads the factor
    of defl_grad_norm first, which waits for it.) `adamw`: further arguments of defl_adamw_step.
    Nothing waits; returns the tensor (norm, factor). A missing gradient under nesterov=True and a list of gradients of the wrong
    length are refused before the counter, the weights or the moments change."""
    rest_grads = list(rest_grads)
    _look_ahead_has_gradients(weights, grads, kw.get("nesterov"))
    sizes = getattr(rest, "sizes", rest_grads)
    if len(sizes) != len(rest_grads):
        raise ValueError("%d gradients for %d parameters" % (len(rest_grads), len(sizes)))
    every = [g for g in grads.values() if g is not None] + [g for g in rest_grads if g is not None]
    clip = ctx.defl_grad_norm(every, max_norm, step=rest_step)
    muon_step_groups(ctx, weights, momenta, grads, lr, mu, window, oversample, power_iters, coeff_schedule, grad_scale=clip, **kw)
    ctx.defl_adamw_step(rest, rest_grads, rest_lr, rest_step, grad_scale=clip, **(adamw or {}))
    return clip
